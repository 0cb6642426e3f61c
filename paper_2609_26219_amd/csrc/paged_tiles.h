// What the kernels of attention load and decode of a paged cache, for one head_dim
// (PKV_HEAD_DIM): the tiles of attend.hip, whose notes give the operands' layouts, and of weigh.hip.
#ifndef PKV_PAGED_TILES_H
#define PKV_PAGED_TILES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "serve.h"

#ifndef PKV_HEAD_DIM
#error "build with -DPKV_HEAD_DIM=64, 128 or 256"
#endif

namespace pkv {
namespace {

constexpr int D = PKV_HEAD_DIM;
constexpr int kChannels = D / 16; // channels of a lane in V, matrix instructions of one O^T update
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

// A nibble or byte becomes a binary16 value by being put into the mantissa of 1024 (units of 1; a nibble four
// bits up into that of 64), and the offset is taken off again with the centre: both exact.  The constants sit
// in registers, where one instruction masks and merges (with literals it takes two).
struct Magic {
  uint32_t low, high, k1024, k64;  // nibble masks, 1024 and 64 in both halves
};
__device__ __forceinline__ Magic magic() {
  Magic m{0x000F000Fu, 0x00F000F0u, 0x64006400u, 0x54005400u};
  asm volatile("" : "+v"(m.low), "+v"(m.high), "+v"(m.k1024), "+v"(m.k64));
  return m;
}
__device__ __forceinline__ uint32_t low_nibbles(const Magic& m, uint32_t w) {
  return add_f16((w & m.low) | m.k1024, -1032.0f);
}
__device__ __forceinline__ uint32_t high_nibbles(const Magic& m, uint32_t w) {
  return add_f16((w & m.high) | m.k64, -72.0f);
}
// Bytes `at` and `at` + 2 of w.
__device__ __forceinline__ uint32_t two_bytes(const Magic& m, uint32_t w, int at) {
  return add_f16(__builtin_amdgcn_perm(w, m.k1024, at ? 0x03070105u : 0x03060104u), -1152.0f);
}

// The K operand of instruction `step` from a lane's words: 8 channels, codes
// centred.  Order of the 8 channels within the operand: 4 bits (0,4)(1,5)(2,6)(3,7), 8 bits
// (0,2)(1,3)(4,6)(5,7), 16 bits as they lie.
template <int BITS>
__device__ __forceinline__ u32x4 k_operand(const Magic& m, const uint32_t* w, int step) {
  if constexpr (BITS == 16) {
    return u32x4{w[4 * step], w[4 * step + 1], w[4 * step + 2], w[4 * step + 3]};
  } else if constexpr (BITS == 8) {
    return u32x4{two_bytes(m, w[2 * step], 0), two_bytes(m, w[2 * step], 1), two_bytes(m, w[2 * step + 1], 0),
                 two_bytes(m, w[2 * step + 1], 1)};
  } else {
    const uint32_t b = w[step], h = b >> 8;
    return u32x4{low_nibbles(m, b), high_nibbles(m, b), low_nibbles(m, h), high_nibbles(m, h)};
  }
}

// First channel of the 8 that lane group c has in instruction `step`, where a
// lane loads its part of a row in pieces of up to 16 bytes and the four lanes of a row lie next
// to each other, so that they take 64 bytes of a line together.
template <int BITS>
__device__ __forceinline__ constexpr int k_first(int step, int c) {
  constexpr int kBytes = D / 4 * BITS / 8 < 16 ? D / 4 * BITS / 8 : 16, kPer = kBytes * 8 / BITS, kSteps = kPer / 8;
  return step / kSteps * 4 * kPer + c * kPer + step % kSteps * 8;
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
__device__ __forceinline__ uint32_t v_pair(const Magic& m, const uint32_t* a, const uint32_t* b, int j) {
  if constexpr (BITS == 16) {
    return __builtin_amdgcn_perm(b[j / 2], a[j / 2], j & 1 ? 0x07060302u : 0x05040100u);
  } else if constexpr (BITS == 8) {
    return two_bytes(m, __builtin_amdgcn_perm(b[j / 4], a[j / 4], j & 2 ? 0x07060302u : 0x05040100u), j & 1);
  } else {
    uint32_t w = __builtin_amdgcn_perm(b[j / 8], a[j / 8], j & 4 ? 0x07060302u : 0x05040100u);
    if (j & 2) w >>= 8;
    return j & 1 ? high_nibbles(m, w) : low_nibbles(m, w);
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
// token's keys and of four tokens' values.
template <int BITS>
struct Keys {
  static constexpr int kBytes = D / 4 * BITS / 8;
  uint32_t w[2][kBytes / 4];
};
template <int BITS>
struct Values {
  static constexpr int kBytes = kChannels * BITS / 8, kWords = (kBytes + 3) / 4;
  uint32_t w[2][4][kWords];
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

// Where a segment's cache begins, and where a tile's tokens lie in it.  WHOLE: pages hold 16 slots or more, so each
// half of a tile lies on one page, whose number the wave shares (-1: not there); else every lane looks its tokens up
// (32 ragged sequences over 4 bits: 74 us, join included, on pages of 16; on pages of 8, with every lane's lookups, 271, of
// 1 slot 229).
// Tokens that are not there are read from page 0, which exists.
struct Source {
  const char* k;           // page 0, slot 0 of the head
  const char* v;
  const uint32_t* scales;  // keys'
  const int32_t* table;
};
template <int KB>
__device__ __forceinline__ Source source_of(const ServeArgs& s, int32_t seq, int32_t head) {
  Source f;
  if constexpr (KB == 16) {
    f.k = reinterpret_cast<const char*>(s.k_cache + head * D);
    f.v = reinterpret_cast<const char*>(s.v_cache + head * D);
    f.scales = nullptr;
  } else {
    f.k = reinterpret_cast<const char*>(s.codes + head * s.head_stride);
    f.v = f.k + s.v_offset;
    f.scales = s.scales + ((int64_t(head) * 2) << s.log2P);
  }
  f.table = s.page_table + int64_t(seq) * s.pages_per_seq;
  return f;
}
struct Tile {
  int32_t t0;
  int32_t page[2];  // WHOLE: of each half, or -1
};
// Byte offset of a slot's row, of `row` bytes, on a page (a page is at most 2 GiB, its number 32 bits).
template <int BITS>
__device__ __forceinline__ uint64_t row_at(const ServeArgs& s, int32_t page, uint32_t slot, uint32_t row) {
  const uint32_t stride = uint32_t(s.page_stride) * (BITS == 16 ? 2 : 1);
  return uint64_t(uint32_t(page < 0 ? 0 : page)) * stride + uint64_t(slot) * row;
}

template <int BITS, bool WHOLE>
__device__ __forceinline__ void load_keys(const ServeArgs& s, const Source& f, const Tile& tile, int c, int x,
                                          Keys<BITS>& p) {
  constexpr int kPiece = Keys<BITS>::kBytes < 16 ? Keys<BITS>::kBytes : 16;
  const int32_t slots = (1 << s.log2P) - 1;
  const uint32_t row = BITS == 16 ? uint32_t(s.H) * D * 2 : D * BITS / 8, mine = c * kPiece;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int32_t t = tile.t0 + 16 * u;
    if constexpr (WHOLE) {
      const char* from = f.k + row_at<BITS>(s, tile.page[u], t & slots, row);
#pragma unroll
      for (int n = 0; n < Keys<BITS>::kBytes / kPiece; ++n)
        load_at<kPiece>(p.w[u] + n * (kPiece / 4), from + n * (4 * kPiece), x * row + mine);
    } else {
      const char* from = f.k + row_at<BITS>(s, page_of(s, f.table, (t + x) >> s.log2P), (t + x) & slots, row) + mine;
#pragma unroll
      for (int n = 0; n < Keys<BITS>::kBytes / kPiece; ++n)
        load_bytes<kPiece>(p.w[u] + n * (kPiece / 4), from + n * (4 * kPiece));
    }
  }
}

template <int BITS, bool WHOLE>
__device__ __forceinline__ void load_values(const ServeArgs& s, const Source& f, const Tile& tile, int c, int x,
                                            Values<BITS>& p) {
  const int32_t slots = (1 << s.log2P) - 1;
  const uint32_t row = BITS == 16 ? uint32_t(s.H) * D * 2 : D * BITS / 8, mine = x * Values<BITS>::kBytes;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int32_t t = tile.t0 + 16 * u;
    if constexpr (WHOLE) {
      const char* from = f.v + row_at<BITS>(s, tile.page[u], t & slots, row);
#pragma unroll
      for (int i = 0; i < 4; ++i) load_at<Values<BITS>::kBytes>(p.w[u][i], from + i * row, 4 * c * row + mine);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int32_t tok = t + 4 * c + i;
        load_bytes<Values<BITS>::kBytes>(
            p.w[u][i], f.v + row_at<BITS>(s, page_of(s, f.table, tok >> s.log2P), tok & slots, row) + mine);
      }
    }
  }
}

// The tile's 64 (scale, zero) words, one to a lane: keys' of its 32 tokens, then values'.
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_scale(const ServeArgs& s, const Source& f, const Tile& tile, int lane) {
  const int32_t slots = (1 << s.log2P) - 1, t = tile.t0 + (lane & 31);
  const int32_t page = WHOLE ? (lane & 16 ? tile.page[1] : tile.page[0]) : page_of(s, f.table, t >> s.log2P);
  return f.scales[uint64_t(uint32_t(page < 0 ? 0 : page)) * uint32_t(s.scale_stride) +
                  ((uint32_t(lane >> 5) << s.log2P) + uint32_t(t & slots))];
}

// Which of the lane's tokens are there: bit 4u + i for token t0 + 16u + 4c + i.
template <bool WHOLE>
__device__ __forceinline__ uint32_t tokens_there(const ServeArgs& s, const Source& f, const Tile& tile, int c) {
  if constexpr (WHOLE) return (tile.page[0] >= 0 ? 0x0Fu : 0u) | (tile.page[1] >= 0 ? 0xF0u : 0u);
  uint32_t there = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      there |= (page_of(s, f.table, (tile.t0 + 16 * u + 4 * c + i) >> s.log2P) >= 0 ? 1u : 0u) << (4 * u + i);
  return there;
}

// What a row sees: tokens t <= hi with t > lo or t < sinks.
struct Sight {
  int32_t hi, lo;
};

// Entry `at` of a table that the wave shares, by a scalar load.
__device__ __forceinline__ int32_t scalar_entry(const int32_t* table, int32_t at) {
  const auto* t = (const __attribute__((address_space(4))) int32_t*)(reinterpret_cast<uintptr_t>(table));
  return t[__builtin_amdgcn_readfirstlane(at)];
}

}  // namespace
}  // namespace pkv

#endif  // PKV_PAGED_TILES_H
