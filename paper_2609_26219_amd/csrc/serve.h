// The serving calls (pkv_cache_append, pkv_cache_read, pkv_attention): what
// their host checks hand to the kernels.
#ifndef PKV_SERVE_H
#define PKV_SERVE_H

#include <stddef.h>
#include <stdint.h>

#include "pkv.h"
#include "pkv_internal.h"

namespace pkv {

// One layer's cache and the rows of a call, as the kernels see them.
struct ServeArgs {
  const int32_t* token_start;
  const int32_t* kv_lens;
  const int32_t* positions;
  const int32_t* page_table;
  // FP16 tag: the layer's first slot of K and of V, in 16-bit elements; a page
  // is page_stride elements after the one before, a slot H * D.
  uint16_t* k_cache;
  uint16_t* v_cache;
  // Quantised tags: the layer's codes (bytes) and (scale, zero) words; a page
  // is page_stride bytes / scale_stride words after the one before, a head
  // head_stride bytes / 2 * P words, the V tile v_offset bytes after the K tile.
  uint8_t* codes;
  uint32_t* scales;
  int64_t page_stride;
  int64_t scale_stride;
  int64_t head_stride;
  int64_t v_offset;
  int64_t pool_pages;
  int32_t num_seqs, num_tokens, max_tokens, pages_per_seq;
  int32_t max_kv;  // bound of kv_lens, at most pages_per_seq * P
  int32_t log2P;
  int32_t H, D;
  int32_t tag, bf16;
};

// A sequence's rows [start, start + count) of a call and its tokens in the cache; the last row is `trail` rows on from the first.
struct SequenceRows {
  int32_t start, count, kv_len, trail;
};

// From what the device's arrays hold, whatever that is (constexpr: for the kernels and the host's tests).
constexpr SequenceRows rows_of_sequence(const ServeArgs& s, int32_t start, int32_t end, int32_t kv_len) {
  SequenceRows r{};
  r.start = start < 0 ? 0 : start < s.num_tokens ? start : s.num_tokens;
  end = end < 0 ? 0 : end < s.num_tokens ? end : s.num_tokens;
  r.trail = end - r.start;
  r.count = r.trail < s.max_tokens ? r.trail : s.max_tokens;
  r.kv_len = kv_len < 0 ? 0 : kv_len < s.max_kv ? kv_len : s.max_kv;
  return r;
}

struct RowArgs {
  uint16_t* k;
  uint16_t* v;
  int64_t token_stride, head_stride;
};

struct AttendArgs {
  const uint16_t* q;
  uint16_t* out;
  float* lse;         // or null
  // Parts of rows: [..][D] sums relative to a reference, and [..][2] the reference (base 2) and the sum of the
  // probabilities.  Splits: [num_tokens * Hq][splits]; pieces: [pieces][H][part_rows].
  float* part;
  float* part_ml;
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
  int32_t Hq, group;  // query heads, query heads per KV head
  int32_t window, sinks;
  float scale;        // scale * log2(e)
  int32_t tiles;      // row tiles of a workgroup
  int32_t row_tiles;  // workgroups' shares of the rows of one sequence and KV head
  int32_t splits;     // many rows: workgroups that share the tokens of a row tile
  int32_t pieces;     // few rows: most pieces of all sequences' tokens together (0: each sequence is whole)
  int32_t part_rows;  // rows of a sequence and KV head
  int32_t chunk;      // least tiles of tokens in a split or piece
};

// How an attention call is launched.
struct AttendLaunch {
  int32_t tiles, row_tiles, splits, pieces, part_rows, chunk;
  int64_t groups;           // workgroups
  uint64_t part_bytes;      // of AttendArgs::part, then part_ml
  uint64_t workspace_bytes; // both
};

// A launch has fewer than 2^32 threads, in workgroups of 256.
constexpr int64_t kMostGroups = int64_t(1) << 24;

constexpr int kRowTile = 16;   // rows (token, query head of one KV head) of a matrix instruction
constexpr int kTokenTile = 32; // cached tokens a wave takes at a time

// Of few rows, up to few_tiles row tiles are shared by a workgroup's waves, which deal the tokens among themselves; many
// rows are dealt to them, many_tiles row tiles to a workgroup, and the tokens shared: kManyElems keys and as many values
// at a time.  (A wave's queries and sums take 6 registers a row of 128 channels: two row tiles leave room for two waves a SIMD.)
constexpr int few_tiles(int head_dim) { return head_dim > 128 ? 1 : 2; }
constexpr int many_tiles(int head_dim) { return 4 * few_tiles(head_dim); }
constexpr int kManyElems = 8192;
// Rows of a sequence and KV head, in workgroups' shares of few rows, above which they are many.  32 ragged sequences of up
// to 16384 tokens, 8 heads of 128, 4 bits, us with few | many: 32 rows 115 | 270, 64 rows 207 | 311, 96 rows 289 | 327, and
// 128 rows would be four shares of 97.  16-bit caches, 64 rows: 334 | 332.
constexpr int few_shares(int key_bits) { return key_bits == 16 ? 1 : 3; }
// Sequences of few rows and no more tiles of tokens are not cut, which saves the second kernel: 8 heads, a sequence
// of 700 tokens 11.6 us against 9.6 + 4.4, of 1500 tokens 17.0 against 9.4 + 4.4.  Where the sequences alone give a
// compute unit its workgroup, up to kWholeTilesOfMany: 32 of 2000 tokens 25.3 against 23.6 + 6.6.
constexpr int kWholeTiles = 28;
constexpr int kWholeTilesOfMany = 64;

// Host checks that need no GPU; they fill the arguments.
pkv_status_t serve_args(const pkv_model_t* model, const pkv_paged_cache_t* cache, const pkv_batch_t* batch,
                        bool pointers, ServeArgs* out);
pkv_status_t row_args(const ServeArgs& s, const void* k, const void* v, int64_t token_stride, int64_t head_stride,
                      RowArgs* out);
pkv_status_t attend_args(const ServeArgs& s, const pkv_attention_t* a, bool pointers, AttendArgs* out);
AttendLaunch attend_launch(const ServeArgs& s, const AttendArgs& a);

}  // namespace pkv

#endif  // PKV_SERVE_H
