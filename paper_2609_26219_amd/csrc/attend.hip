// Attention over a paged cache (pkv_attention), for one head_dim
// (PKV_HEAD_DIM; built once for each of 64, 128 and 256).
//
// A workgroup takes one row tile: kRowTile rows of one sequence and KV head, a row
// being a token of the call and one of the query heads that share the KV head, so
// that every cached row is loaded and decoded once for all of them.  The tiles of kTokenTile
// cached tokens that some row sees are dealt to `splits` workgroups, and a
// workgroup's to its four waves.  A wave keeps the running maximum and sum of the
// softmax and joins them with the others' at the end: one pass over the
// cache.
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
// two that keeps the largest near 2^14, so that small scales lose nothing).
// Queries go in as binary16 too, each row scaled by a power of two.  16-bit caches use the
// matrix instructions of their own type, p_t rounded to it.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "pkv.h"
#include "pkv_internal.h"
#include "serve.h"

#ifndef PKV_HEAD_DIM
#error "build with -DPKV_HEAD_DIM=64, 128 or 256"
#endif

namespace pkv {
namespace {

constexpr int D = PKV_HEAD_DIM;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kQkSteps = D / 32;  // matrix instructions of one S^T
constexpr int kChannels = D / 16; // channels of a lane in V, matrix instructions of one O^T update
constexpr int kMostRowTiles = most_row_tiles(D);
constexpr float kInf = __builtin_inff();

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float f16_float(uint32_t bits) {
  return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
}
__device__ __forceinline__ float bf16_float(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), f16x2));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}
__device__ __forceinline__ uint32_t add_f16(uint32_t a, float b) {
  const _Float16 h = static_cast<_Float16>(b);
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, a) + f16x2{h, h});
}
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// BYTES consecutive bytes into registers (BYTES 2: the low half of one).
template <int BYTES>
__device__ __forceinline__ void load_bytes(uint32_t* to, const void* from) {
  if constexpr (BYTES >= 16) {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const u32x4 w = static_cast<const u32x4*>(from)[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) to[4 * i + e] = w[e];
    }
  } else if constexpr (BYTES == 8) {
    const u32x2 w = *static_cast<const u32x2*>(from);
    to[0] = w[0];
    to[1] = w[1];
  } else if constexpr (BYTES == 4) {
    to[0] = *static_cast<const uint32_t*>(from);
  } else {
    static_assert(BYTES == 2, "a lane's piece");
    to[0] = *static_cast<const uint16_t*>(from);
  }
}

// The K operand of instruction `step` from a lane's words: 8 channels, codes
// centred.  Order of the 8 channels within the operand: 4 bits (0,4)(1,5)(2,6)(3,7), 8 bits
// (0,2)(1,3)(4,6)(5,7), 16 bits as they lie.  A nibble or byte becomes a binary16
// value by or-ing it into the mantissa of 1024 (units of 1; a nibble four bits
// up into that of 64), and the offset is taken off again with the centre: both exact.
template <int BITS>
__device__ __forceinline__ u32x4 k_operand(const uint32_t* w, int step) {
  if constexpr (BITS == 16) {
    return u32x4{w[4 * step], w[4 * step + 1], w[4 * step + 2], w[4 * step + 3]};
  } else if constexpr (BITS == 8) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t b = w[2 * step + i];
      r[2 * i] = add_f16((b & 0x00FF00FFu) | 0x64006400u, -1152.0f);
      r[2 * i + 1] = add_f16(((b >> 8) & 0x00FF00FFu) | 0x64006400u, -1152.0f);
    }
    return r;
  } else {
    const uint32_t b = w[step], h = b >> 8;
    return u32x4{add_f16((b & 0x000F000Fu) | 0x64006400u, -1032.0f), add_f16((b & 0x00F000F0u) | 0x54005400u, -72.0f),
                 add_f16((h & 0x000F000Fu) | 0x64006400u, -1032.0f), add_f16((h & 0x00F000F0u) | 0x54005400u, -72.0f)};
  }
}

// Channel e (0..7) of register pair position p in the order above.
template <int BITS>
__device__ __forceinline__ constexpr int k_channel(int p, int half) {
  if (BITS == 16) return 2 * p + half;
  if (BITS == 8) return (p >> 1) * 4 + (p & 1) + 2 * half;
  return p + 4 * half;
}

// One channel of two tokens as a packed pair, from the tokens' words a and b of the
// lane's V pieces; j counts the lane's channels.
template <int BITS>
__device__ __forceinline__ uint32_t v_pair(const uint32_t* a, const uint32_t* b, int j) {
  if constexpr (BITS == 16) {
    return __builtin_amdgcn_perm(b[j / 2], a[j / 2], j & 1 ? 0x07060302u : 0x05040100u);
  } else if constexpr (BITS == 8) {
    const uint32_t w = __builtin_amdgcn_perm(b[j / 4], a[j / 4], j & 2 ? 0x07060302u : 0x05040100u);
    return add_f16(((j & 1 ? w >> 8 : w) & 0x00FF00FFu) | 0x64006400u, -1152.0f);
  } else {
    uint32_t w = __builtin_amdgcn_perm(b[j / 8], a[j / 8], j & 4 ? 0x07060302u : 0x05040100u);
    if (j & 2) w >>= 8;
    return j & 1 ? add_f16((w & 0x00F000F0u) | 0x54005400u, -72.0f)
                 : add_f16((w & 0x000F000Fu) | 0x64006400u, -1032.0f);
  }
}

// Sums and maxima over the four lanes (c) of a column: the halves of the wave
// exchanged, then the neighbouring rows of 16 lanes.
__device__ __forceinline__ float over_c_max(float v) {
  u32x2 w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __builtin_fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
  w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __builtin_fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float over_c_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}
__device__ __forceinline__ int over_x_max(int v) {
  for (int off = 1; off < 16; off <<= 1) v = max(v, __shfl_xor(v, off));
  return v;
}
__device__ __forceinline__ int over_x_min(int v) {
  for (int off = 1; off < 16; off <<= 1) v = min(v, __shfl_xor(v, off));
  return v;
}

// What a tile's lane holds of the cache: for each half of 16 tokens its piece of one
// token's keys, of four tokens' values, and those four tokens' (scale, zero).
template <int BITS>
struct Keys {
  static constexpr int kBytes = D / 4 * BITS / 8;
  uint32_t w[2][kBytes / 4];
  uint32_t scale[2][4];
};
template <int BITS>
struct Values {
  static constexpr int kBytes = kChannels * BITS / 8, kWords = (kBytes + 3) / 4;
  uint32_t w[2][4][kWords];
  uint32_t scale[2][4];
};

// Physical page of a logical one, or -1.
__device__ __forceinline__ int32_t page_of(const ServeArgs& s, const int32_t* table, int32_t at) {
  if (at >= s.pages_per_seq) return -1;
  const int32_t p = table[at];
  return p >= 0 && p < s.pool_pages ? p : -1;
}

// Bytes into a lane's piece from a base that the wave shares.
template <int BYTES>
__device__ __forceinline__ void load_at(uint32_t* to, const void* base, uint32_t off) {
  load_bytes<BYTES>(to, static_cast<const char*>(base) + off);
}

// Load the keys or values of the tile of tokens [t0, t0 + 32); tokens that are not
// there are loaded from page 0, which exists.  WHOLE: pages hold 16 slots or more, so
// each half of the tile lies on one page (`pages`, or -1).
template <int BITS, bool WHOLE>
__device__ __forceinline__ void load_keys(const ServeArgs& s, const int32_t* table, int head, int32_t t0,
                                          const int32_t (&pages)[2], int c, int x, Keys<BITS>& p) {
  const int32_t slots = (1 << s.log2P) - 1;
  const uint32_t row = BITS == 16 ? uint32_t(s.H) * D * 2 : D * BITS / 8, mine = c * Keys<BITS>::kBytes;
  auto first_of = [&](int64_t page) -> const char* {
    if constexpr (BITS == 16) return reinterpret_cast<const char*>(s.k_cache + page * s.page_stride + head * D);
    return reinterpret_cast<const char*>(s.codes + page * s.page_stride + head * s.head_stride);
  };
  auto scales_of = [&](int64_t page) { return s.scales + page * s.scale_stride + ((int64_t(head) * 2) << s.log2P); };
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int32_t t = t0 + 16 * u;
    if constexpr (WHOLE) {
      const int32_t page = pages[u] >= 0 ? pages[u] : 0;
      const int64_t slot = t & slots;
      load_at<Keys<BITS>::kBytes>(p.w[u], first_of(page) + slot * row, x * row + mine);
      if constexpr (BITS != 16) load_at<16>(p.scale[u], scales_of(page) + slot, 16 * c);
    } else {
      const int32_t page = page_of(s, table, (t + x) >> s.log2P);
      load_bytes<Keys<BITS>::kBytes>(p.w[u], first_of(page >= 0 ? page : 0) + int64_t((t + x) & slots) * row + mine);
      if constexpr (BITS != 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int32_t tok = t + 4 * c + i, at = page_of(s, table, tok >> s.log2P);
          p.scale[u][i] = scales_of(at >= 0 ? at : 0)[tok & slots];
        }
      }
    }
  }
}

template <int BITS, bool WHOLE>
__device__ __forceinline__ void load_values(const ServeArgs& s, const int32_t* table, int head, int32_t t0,
                                            const int32_t (&pages)[2], int c, int x, Values<BITS>& p) {
  const int32_t slots = (1 << s.log2P) - 1;
  const uint32_t row = BITS == 16 ? uint32_t(s.H) * D * 2 : D * BITS / 8, mine = x * Values<BITS>::kBytes;
  auto first_of = [&](int64_t page) -> const char* {
    if constexpr (BITS == 16) return reinterpret_cast<const char*>(s.v_cache + page * s.page_stride + head * D);
    return reinterpret_cast<const char*>(s.codes + page * s.page_stride + head * s.head_stride + s.v_offset);
  };
  auto scales_of = [&](int64_t page) { return s.scales + page * s.scale_stride + ((int64_t(head) * 2 + 1) << s.log2P); };
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int32_t t = t0 + 16 * u;
    if constexpr (WHOLE) {
      const int32_t page = pages[u] >= 0 ? pages[u] : 0;
      const int64_t slot = t & slots;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        load_at<Values<BITS>::kBytes>(p.w[u][i], first_of(page) + (slot + i) * row, 4 * c * row + mine);
      if constexpr (BITS != 16) load_at<16>(p.scale[u], scales_of(page) + slot, 16 * c);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t tok = t + 4 * c + i, at = page_of(s, table, tok >> s.log2P);
        const int64_t slot = tok & slots, page = at >= 0 ? at : 0;
        load_bytes<Values<BITS>::kBytes>(p.w[u][i], first_of(page) + slot * row + mine);
        if constexpr (BITS != 16) p.scale[u][i] = scales_of(page)[slot];
      }
    }
  }
}

// Which of the lane's tokens are there: bit 4u + i for token t0 + 16u + 4c + i.
template <bool WHOLE>
__device__ __forceinline__ uint32_t tokens_there(const ServeArgs& s, const int32_t* table, int32_t t0,
                                                 const int32_t (&pages)[2], int c) {
  if constexpr (WHOLE) return (pages[0] >= 0 ? 0x0Fu : 0u) | (pages[1] >= 0 ? 0xF0u : 0u);
  uint32_t there = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      there |= (page_of(s, table, (t0 + 16 * u + 4 * c + i) >> s.log2P) >= 0 ? 1u : 0u) << (4 * u + i);
  return there;
}

// What a row sees: tokens t <= hi with t > lo or t < sinks.
struct Sight {
  int32_t hi, lo;
};

struct Span {  // of a row tile, over its rows
  int32_t hi_most, hi_least, lo_most, lo_least;
  int32_t sink_tiles, first, tiles;  // tiles of tokens to look at: the sinks', then those from token `first` on
};

// The running softmax of a wave over its rows (lane: row x of each of RT row tiles).
template <int RT>
struct Running {
  f32x4 o[RT][kChannels];
  float ref[RT];   // exponents are taken relative to it (base 2): within kSlack of the largest so far; -inf at first
  float l[RT], o_zero[RT];
  float fac;       // codes: O counts in units of 1 / fac
  float most_scale;
};

// P is stored as 2^kShift p where the operands are binary16, which keeps small
// probabilities clear of its subnormals; the reference of the exponents is moved only
// when a score passes it by kSlack, so that O is rescaled once or twice a row and not
// at every new maximum (with 64 rows in a wave nearly every tile has one).  2^(kShift + kSlack) is
// in binary16's range.
constexpr float kSlack = 8.0f;
constexpr float kShiftOfHalf = 6.0f;

// One tile: `there` of its tokens exist; more_keys and more_values load the next
// tile's over this one's as soon as those have been used.
template <bool BF16, int KB, int VB, int RT, typename MoreKeys, typename MoreValues>
__device__ __forceinline__ void attend_tile(const AttendArgs& a, const Span& span, const Sight (&see)[RT],
                                            const u32x4 (&q)[RT][kQkSteps], const float (&q_sum)[RT],
                                            const float (&f)[RT], int c, int32_t t0, uint32_t there, Keys<KB>& keys,
                                            Values<VB>& values, Running<RT>& st, MoreKeys more_keys,
                                            MoreValues more_values) {
  constexpr bool kCodes = KB != 16;
  constexpr bool kHalf = kCodes || !BF16;  // operands in binary16
  const bool all = t0 + kTokenTile - 1 <= span.hi_least && (span.lo_most < t0 || t0 + kTokenTile <= a.sinks) &&
                   __all(there == 0xFFu);
  // S^T, in units of 1 / f.
  f32x4 t[RT][2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
#pragma unroll
    for (int r = 0; r < RT; ++r) t[r][u] = f32x4{};
#pragma unroll
    for (int i = 0; i < kQkSteps; ++i) {
      const u32x4 k = k_operand<KB>(keys.w[u], i);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if constexpr (kHalf)
          t[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, k),
                                                           __builtin_bit_cast(f16x8, q[r][i]), t[r][u], 0, 0, 0);
        else
          t[r][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k),
                                                            __builtin_bit_cast(bf16x8, q[r][i]), t[r][u], 0, 0, 0);
      }
    }
  }
  float vs[2][4], vz[2][4];
  if constexpr (kCodes) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float sc = f16_float(keys.scale[u][i]);
        const float zc = __builtin_fmaf(sc, float(1 << (KB - 1)), f16_float(keys.scale[u][i] >> 16));
#pragma unroll
        for (int r = 0; r < RT; ++r) t[r][u][i] = __builtin_fmaf(sc, t[r][u][i], zc * q_sum[r]);
        vs[u][i] = f16_float(values.scale[u][i]);
        vz[u][i] = __builtin_fmaf(vs[u][i], float(1 << (VB - 1)), f16_float(values.scale[u][i] >> 16));
      }
  }
  more_keys();
  if (!all) {
    // A row's score where it does not see; the values of tokens that no row sees, whatever lies there.
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t tok = t0 + 16 * u + 4 * c + i;
        const bool is = (there >> (4 * u + i)) & 1;
#pragma unroll
        for (int r = 0; r < RT; ++r)
          t[r][u][i] = is && tok <= see[r].hi && (tok > see[r].lo || tok < a.sinks) ? t[r][u][i] : -kInf;
        const bool any = is && tok <= span.hi_most && (tok > span.lo_least || tok < a.sinks);
        if constexpr (kCodes) {
          vs[u][i] = any ? vs[u][i] : 0.0f;
          vz[u][i] = any ? vz[u][i] : 0.0f;
        } else {
#pragma unroll
          for (int w = 0; w < Values<VB>::kWords; ++w) values.w[u][i][w] = any ? values.w[u][i][w] : 0;
        }
      }
  }
  // The reference of the exponents.
  float top[RT];
  bool move = false;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    top[r] = t[r][0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) top[r] = __builtin_fmaxf(top[r], t[r][u][i]);
    top[r] *= f[r];
    move |= top[r] > st.ref[r] + kSlack;
  }
  if (__any(move)) {
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
  if constexpr (kCodes) {
    float tile_most = vs[0][0];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) tile_most = __builtin_fmaxf(tile_most, vs[u][i]);
    if (__any(tile_most > st.most_scale)) {
      st.most_scale = __builtin_fmaxf(st.most_scale, over_c_max(tile_most));
      // 2^e > the largest scale so far: scales times fac stay below 2^kShift.
      const int e = int(__float_as_uint(st.most_scale) >> 23) - 126;
      const float next = __uint_as_float(uint32_t(127 + int(kShiftOfHalf) - e) << 23);
      if (next != st.fac) {
        const float ratio = next / st.fac;
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int j = 0; j < kChannels; ++j) st.o[r][j] *= ratio;
        st.fac = next;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) vs[u][i] *= st.fac;
  }
  // The probabilities and their sum.
  u32x4 pt[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float base = (kCodes || !kHalf ? 0.0f : kShiftOfHalf) - (st.ref[r] == -kInf ? 0.0f : st.ref[r]);
    float pr[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pr[u][i] = exp2_of(__builtin_fmaf(t[r][u][i], f[r], base));
        st.l[r] += pr[u][i];
        if constexpr (kCodes) {
          st.o_zero[r] = __builtin_fmaf(pr[u][i], vz[u][i], st.o_zero[r]);
          pr[u][i] *= vs[u][i];
        }
      }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        pt[r][2 * u + i] = kHalf ? pack_f16(pr[u][2 * i], pr[u][2 * i + 1]) : pack_bf16(pr[u][2 * i], pr[u][2 * i + 1]);
  }
#pragma unroll
  for (int j = 0; j < kChannels; ++j) {
    u32x4 v;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 2; ++i) v[2 * u + i] = v_pair<VB>(values.w[u][2 * i], values.w[u][2 * i + 1], j);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      if constexpr (kHalf)
        st.o[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, v), __builtin_bit_cast(f16x8, pt[r]),
                                                            st.o[r][j], 0, 0, 0);
      else
        st.o[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v),
                                                             __builtin_bit_cast(bf16x8, pt[r]), st.o[r][j], 0, 0, 0);
    }
  }
  more_values();
}

// Entry `at` of a table that the wave shares, by a scalar load.
__device__ __forceinline__ int32_t scalar_entry(const int32_t* table, int32_t at) {
  const auto* t = (const __attribute__((address_space(4))) int32_t*)(reinterpret_cast<uintptr_t>(table));
  return t[__builtin_amdgcn_readfirstlane(at)];
}

template <bool BF16, int KB, int VB, bool WHOLE, int RT>
__global__ __launch_bounds__(kThreads, RT * D > 256 ? 1 : 2) void attend_kernel(ServeArgs s, AttendArgs a) {
  constexpr bool kCodes = KB != 16;
  constexpr int kRows = kRowTile * RT;
  __shared__ float join_ml[kWaves][kRowTile][2];
  __shared__ float join[kWaves][kRowTile][D + 4];

  uint32_t b = blockIdx.x;
  const int32_t head = int32_t(b % uint32_t(s.H));
  b /= uint32_t(s.H);
  const int32_t split = int32_t(b % uint32_t(a.splits));
  b /= uint32_t(a.splits);
  const int32_t tile = int32_t(b % uint32_t(a.row_tiles));
  const int32_t seq = int32_t(b / uint32_t(a.row_tiles));

  const int lane = threadIdx.x & 63, c = lane >> 4, x = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // The tile's rows.
  int32_t start = scalar_entry(s.token_start, seq), end = scalar_entry(s.token_start, seq + 1);
  int32_t kv_len = scalar_entry(s.kv_lens, seq);
  start = start < 0 ? 0 : start;
  end = end < s.num_tokens ? end : s.num_tokens;
  const int32_t count = end - start < s.max_tokens ? end - start : s.max_tokens;
  const int64_t row0 = int64_t(tile) * kRows;
  if (row0 >= int64_t(count) * a.group) return;  // the whole workgroup
  kv_len = kv_len < 0 ? 0 : kv_len < s.max_kv ? kv_len : s.max_kv;
  Sight see[RT];
  Span span{-1, 0x7FFFFFFF, -1, 0x7FFFFFFF, 0, 0, 0};
  u32x4 q[RT][kQkSteps];
  float q_sum[RT], f[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const uint32_t row = uint32_t(row0) + kRowTile * r + x;
    const int32_t token = int32_t(row / uint32_t(a.group)), sub = int32_t(row % uint32_t(a.group));
    const bool on = token < count;
    see[r] = Sight{-1, -1};
    if (on) {
      const int32_t pos = s.positions ? s.positions[start + token] : kv_len - (end - start) + token;
      see[r].hi = pos < kv_len ? pos : kv_len - 1;
      see[r].hi = see[r].hi < -1 ? -1 : see[r].hi;
      see[r].lo = a.window > 0 && pos >= a.window ? pos - a.window : -1;
      span.hi_least = span.hi_least < see[r].hi ? span.hi_least : see[r].hi;
      if (see[r].hi >= 0 && see[r].lo < span.lo_least) span.lo_least = see[r].lo;
    }
    span.hi_most = span.hi_most > see[r].hi ? span.hi_most : see[r].hi;
    span.lo_most = span.lo_most > see[r].lo ? span.lo_most : see[r].lo;

    // The queries, in the operands' order, and their sum.
    q_sum[r] = 0.0f;
    f[r] = a.scale;
    const uint16_t* from_q = a.q + int64_t(start + token) * a.q_token_stride +
                             int64_t(head * a.group + sub) * a.q_head_stride + c * (D / 4);
    float v[kQkSteps][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kQkSteps; ++i) {
      u32x4 w{};
      if (on) w = *reinterpret_cast<const u32x4*>(from_q + 8 * i);
      if constexpr (!kCodes) {
        q[r][i] = w;
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
      f[r] *= __uint_as_float(uint32_t(127 + e) << 23);
#pragma unroll
      for (int i = 0; i < kQkSteps; ++i) {
#pragma unroll
        for (int p = 0; p < 4; ++p)
          q[r][i][p] = pack_f16(v[i][k_channel<KB>(p, 0)] * down, v[i][k_channel<KB>(p, 1)] * down);
#pragma unroll
        for (int e2 = 0; e2 < 8; ++e2) q_sum[r] += v[i][e2] * down;
      }
      q_sum[r] = over_c_sum(q_sum[r]);
    }
  }
  span.hi_most = __builtin_amdgcn_readfirstlane(over_x_max(span.hi_most));
  span.hi_least = __builtin_amdgcn_readfirstlane(over_x_min(span.hi_least));
  span.lo_most = __builtin_amdgcn_readfirstlane(over_x_max(span.lo_most));
  span.lo_least = __builtin_amdgcn_readfirstlane(over_x_min(span.lo_least));
  if (span.hi_most >= 0) {
    span.first = (span.lo_least + 1) & ~(kTokenTile - 1);
    const int32_t sinks = a.sinks < span.hi_most + 1 ? a.sinks : span.hi_most + 1;
    span.sink_tiles = (sinks + kTokenTile - 1) / kTokenTile;
    span.sink_tiles = span.sink_tiles < span.first / kTokenTile ? span.sink_tiles : span.first / kTokenTile;
    // (a position past kv_lens may leave a row its sinks alone)
    span.tiles = span.sink_tiles + (span.hi_most >= span.first ? (span.hi_most - span.first) / kTokenTile + 1 : 0);
  }
  // This workgroup's share of them.
  int32_t share = (span.tiles + a.splits - 1) / a.splits;
  share = share > a.chunk ? share : a.chunk;
  const int64_t from = int64_t(split) * share;
  const int32_t upto = int32_t(from + share < span.tiles ? from + share : span.tiles);

  const int32_t* table = s.page_table + int64_t(seq) * s.pages_per_seq;
  Running<RT> st;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    st.ref[r] = -kInf;
    st.l[r] = st.o_zero[r] = 0.0f;
#pragma unroll
    for (int j = 0; j < kChannels; ++j) st.o[r][j] = f32x4{};
  }
  st.fac = 1.0f;
  st.most_scale = 0.0f;

  auto tile_at = [&](int32_t it) {
    return it < span.sink_tiles ? it * kTokenTile : span.first + (it - span.sink_tiles) * kTokenTile;
  };
  auto pages_at = [&](int32_t it, int32_t (&pages)[2]) {  // of a tile that exists, else -1
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int32_t at = (tile_at(it) + 16 * u) >> s.log2P;
      pages[u] = WHOLE && it < upto && at < s.pages_per_seq ? scalar_entry(table, at) : -1;
      pages[u] = pages[u] < s.pool_pages ? pages[u] : -1;
    }
  };
  // A tile's keys are loaded while the softmax and the sums of the one before run, its values while its own
  // scores are computed, its pages one tile earlier.
  int32_t it = int32_t(from) + wave;
  if (it < upto) {
    Keys<KB> keys;
    Values<VB> values;
    int32_t pages[2], next[2];
    pages_at(it, pages);
    load_keys<KB, WHOLE>(s, table, head, tile_at(it), pages, c, x, keys);
    load_values<VB, WHOLE>(s, table, head, tile_at(it), pages, c, x, values);
    pages_at(it + kWaves, next);
    for (; it < upto; it += kWaves) {
      const int32_t t0 = tile_at(it), t1 = tile_at(it + kWaves);
      const bool more = it + kWaves < upto;
      const uint32_t there = tokens_there<WHOLE>(s, table, t0, pages, c);
      attend_tile<BF16, KB, VB, RT>(
          a, span, see, q, q_sum, f, c, t0, there, keys, values, st,
          [&] {
            if (more) load_keys<KB, WHOLE>(s, table, head, t1, next, c, x, keys);
          },
          [&] {
            if (more) load_values<VB, WHOLE>(s, table, head, t1, next, c, x, values);
          });
      pages[0] = next[0];
      pages[1] = next[1];
      pages_at(it + 2 * kWaves, next);
    }
  }

  // Join the waves, a row tile at a time: every one's sums relative to the largest reference.
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = over_c_sum(st.l[r]), m = st.ref[r];
    const float o_zero = kCodes ? over_c_sum(st.o_zero[r]) : 0.0f;
    if (r) __syncthreads();
    if (c == 0) {
      join_ml[wave][x][0] = m;
      join_ml[wave][x][1] = l;
    }
    __syncthreads();
    float m_all = -kInf;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m_all = __builtin_fmaxf(m_all, join_ml[w][x][0]);
    const float part = m == -kInf ? 0.0f : exp2_of(m - m_all);
    const float unit = kCodes ? part / st.fac : part;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < kChannels; ++j)
        join[wave][x][(4 * c + i) * kChannels + j] =
            m == -kInf ? 0.0f : kCodes ? __builtin_fmaf(o_zero, part, st.o[r][j][i] * unit) : st.o[r][j][i] * part;
    __syncthreads();
    constexpr int kPerRow = kThreads / kRowTile, kPer = D / kPerRow;  // 16 threads to a row
    const int y = threadIdx.x / kPerRow, at = (threadIdx.x % kPerRow) * kPer;
    const uint32_t out_row = uint32_t(row0) + kRowTile * r + y;
    const int32_t out_token = int32_t(out_row / uint32_t(a.group));
    if (out_token >= count) continue;
    const int32_t out_head = head * a.group + int32_t(out_row % uint32_t(a.group));
    float mm = -kInf, ll = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mm = __builtin_fmaxf(mm, join_ml[w][y][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      ll += join_ml[w][y][0] == -kInf ? 0.0f : join_ml[w][y][1] * exp2_of(join_ml[w][y][0] - mm);
    float sum[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      sum[e] = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum[e] += join[w][y][at + e];
    }
    const int64_t flat = int64_t(start + out_token) * a.Hq + out_head;
    if (a.splits > 1) {
      const int64_t slot = flat * a.splits + split;
#pragma unroll
      for (int e = 0; e < kPer; e += 4)
        *reinterpret_cast<f32x4*>(a.part + slot * D + at + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
      if (at == 0) *reinterpret_cast<f32x2*>(a.part_ml + 2 * slot) = f32x2{mm, ll};
      continue;
    }
    const float inv = ll > 0.0f ? 1.0f / ll : ll == 0.0f ? 0.0f : ll;
    uint32_t word[kPer / 2];
#pragma unroll
    for (int e = 0; e < kPer; e += 2)
      word[e / 2] = s.bf16 ? pack_bf16(sum[e] * inv, sum[e + 1] * inv) : pack_f16(sum[e] * inv, sum[e + 1] * inv);
    uint16_t* to = a.out + int64_t(start + out_token) * a.out_token_stride + int64_t(out_head) * a.out_head_stride + at;
#pragma unroll
    for (int e = 0; e < kPer / 2; e += 2) *reinterpret_cast<u32x2*>(to + 2 * e) = u32x2{word[e], word[e + 1]};
    constexpr float kUp = kCodes || BF16 ? 1.0f : 1.0f / 64.0f;  // l counts 2^kShift to one where p does
    if (a.lse && at == 0)
      a.lse[flat] = ll == 0.0f ? -kInf : (mm + __builtin_amdgcn_logf(ll * kUp)) * 0.69314718055994531f;
  }
}

// Joins the splits of each row: one wave per row.
__global__ __launch_bounds__(kThreads) void join_kernel(ServeArgs s, AttendArgs a, float up) {
  const int lane = threadIdx.x & 63;
  const int64_t flat = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (flat >= int64_t(s.num_tokens) * a.Hq) return;
  const int32_t token = int32_t(flat / a.Hq), head = int32_t(flat % a.Hq);
  // Rows of no sequence have no parts.
  const int32_t first = s.token_start[0], last = s.token_start[s.num_seqs];
  if (token < first || token >= last) return;
  const f32x2* ml = reinterpret_cast<const f32x2*>(a.part_ml) + flat * a.splits;
  float m = -kInf;
  for (int i = lane; i < a.splits; i += 64) m = __builtin_fmaxf(m, ml[i][0]);
  for (int off = 1; off < 64; off <<= 1) m = __builtin_fmaxf(m, __shfl_xor(m, off));
  float l = 0.0f;
  constexpr int kPer = D / 64;
  float sum[kPer] = {};
  for (int i = 0; i < a.splits; ++i) {
    const f32x2 w = ml[i];
    if (w[1] == 0.0f) continue;
    const float scale = exp2_of(w[0] - m);
    l += w[1] * scale;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      sum[e] = __builtin_fmaf(a.part[(flat * a.splits + i) * D + lane * kPer + e], scale, sum[e]);
  }
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  uint16_t* to = a.out + token * a.out_token_stride + head * a.out_head_stride + lane * kPer;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const uint32_t w = s.bf16 ? pack_bf16(sum[e] * inv, 0.0f) : pack_f16(sum[e] * inv, 0.0f);
    to[e] = uint16_t(w);
  }
  if (a.lse && lane == 0) a.lse[flat] = l == 0.0f ? -kInf : (m + __builtin_amdgcn_logf(l * up)) * 0.69314718055994531f;
}

}  // namespace

#define PKV_JOINED2(a, b) a##b
#define PKV_JOINED(a, b) PKV_JOINED2(a, b)

pkv_status_t PKV_JOINED(launch_attend_, PKV_HEAD_DIM)(const ServeArgs& s, const AttendArgs& a, int64_t groups,
                                                      hipStream_t stream) {
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(uint32_t(groups)), dim3(kThreads), 0, stream, s, a); };
  auto by_tag = [&](auto whole, auto tiles) {
    constexpr bool kWhole = decltype(whole)::value;
    constexpr int kTiles = decltype(tiles)::value;
    switch (s.tag) {
      case PKV_TAG_FP16:
        s.bf16 ? go(attend_kernel<true, 16, 16, kWhole, kTiles>) : go(attend_kernel<false, 16, 16, kWhole, kTiles>);
        break;
      case PKV_TAG_K8V8: go(attend_kernel<false, 8, 8, kWhole, kTiles>); break;
      case PKV_TAG_K8V4: go(attend_kernel<false, 8, 4, kWhole, kTiles>); break;
      default: go(attend_kernel<false, 4, 4, kWhole, kTiles>); break;
    }
  };
  auto by_tiles = [&](auto whole) {
    if constexpr (kMostRowTiles >= 4)
      if (a.tiles == 4) return by_tag(whole, std::integral_constant<int, 4>{});
    a.tiles == 2 ? by_tag(whole, std::integral_constant<int, 2>{}) : by_tag(whole, std::integral_constant<int, 1>{});
  };
  s.log2P >= 4 ? by_tiles(std::true_type{}) : by_tiles(std::false_type{});
  if (hipGetLastError() != hipSuccess) return PKV_ERR_DEVICE;
  if (a.splits > 1) {
    const int64_t rows = int64_t(s.num_tokens) * a.Hq;
    const float up = s.tag == PKV_TAG_FP16 && !s.bf16 ? 1.0f / 64.0f : 1.0f;
    hipLaunchKernelGGL(join_kernel, dim3(uint32_t((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0, stream, s, a, up);
    if (hipGetLastError() != hipSuccess) return PKV_ERR_DEVICE;
  }
  return PKV_OK;
}

}  // namespace pkv
