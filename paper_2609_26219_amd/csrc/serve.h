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

// Of a sequence's rows that are the last of its tokens, those [first, end) that see one of tokens [begin, last], with a
// window (0: none) and sinks (a superset: all of the tokens may be between sinks and window).  Always within the rows.
struct RowRange {
  int32_t first, end;
};
constexpr RowRange rows_that_see(const SequenceRows& g, int32_t begin, int32_t last, int32_t window, int32_t sinks) {
  if (g.count <= 0) return RowRange{0, 0};
  const int64_t pos0 = int64_t(g.kv_len) - g.trail;  // of row 0; below zero where rows are more than tokens
  int64_t first = begin - pos0, end = g.count;
  if (window > 0 && begin >= sinks && int64_t(last) + window - pos0 < end) end = int64_t(last) + window - pos0;
  end = end < 0 ? 0 : end;
  first = first < 0 ? 0 : first < end ? first : end;
  return RowRange{int32_t(first), int32_t(end)};
}

struct RowArgs {
  uint16_t* k;
  uint16_t* v;
  int64_t token_stride, head_stride;
};

// Rows turned to their positions, and how.
struct RotateArgs {
  const int32_t* offset;  // of each sequence, or null
  const uint16_t* x;
  uint16_t* out;
  int64_t x_token_stride, x_head_stride, out_token_stride, out_head_stride;
  double amplitude;
  int32_t heads;
  int32_t rotary;       // channels that turn
  int32_t interleaved;  // pairs (2j, 2j + 1), else (j, j + rotary / 2)
  int32_t reserved;
  double freq[kMaxHeadDim / 2];  // of each pair: an argument, so that a call needs no device memory for it
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

struct WeighArgs {
  const uint16_t* q;
  const float* lse;      // [num_tokens][Hq]
  const float* weights;  // before, or null (decay 0)
  float* out;
  float* part;           // [splits][H][num_seqs][max_kv], or null: sums go straight to out
  int64_t q_token_stride, q_head_stride, seq_stride, head_stride;
  float decay;
  float scale;           // scale * log2(e)
  int32_t Hq, group, window, sinks;
  int32_t joint;         // one weight a token, of all heads
  int32_t tiles;         // workgroups along a sequence's tokens
  int32_t chunk, subs;   // few rows: tokens of a workgroup (0: an even share), and the parts that its waves take
  int32_t splits;        // many rows: workgroups that share the rows of a tile of tokens
  int32_t row_tiles;     // most tiles of rows of a sequence,
  int64_t all_tiles;     // and of all of them
  void* rows;            // the tiles, [H][all_tiles]
};

// How a call of weights is launched.
struct WeighLaunch {
  int32_t few_tiles;    // tiles of few rows, or 0: many
  int32_t tiles, chunk, subs, splits, row_tiles;
  int64_t all_tiles, groups, prepare_groups, join_groups;
  uint64_t part_bytes;      // of WeighArgs::part, then rows
  uint64_t workspace_bytes; // both
};

// Of a segment of a long row: its keys that share the first digit of the last one kept, and those of larger digits; then the
// tokens before it that are equal to the last one kept, and above it.
struct KeepSegment {
  int32_t listed, above;
};
struct KeepRow {  // the last key kept (its first digit at first), and how many of those equal to it stay
  uint32_t last, need;
};

// The tokens of each sequence (and head) that stay.
struct KeepArgs {
  const float* weights;
  const int32_t* budgets;  // of each sequence, or null
  int32_t* kept;           // [num_seqs][heads][budget]
  int32_t* kept_lens;
  int64_t seq_stride, head_stride;
  int32_t heads, budget, sinks, recent;
  int32_t segments;        // workgroups of a row, or 0: one
  uint32_t* counts;        // [rows][segments][2048]
  uint32_t* lists;         // [rows][segments][kKeepSegment]
  KeepSegment* segment;    // [rows][segments]
  KeepRow* row;            // [rows]
};

constexpr int kKeepSegment = 8192;  // tokens of a segment
// A choice of up to kFewKeptRows rows that may be longer than kWholeRow is made by segments.  Whole calls, us, by segments | by a
// workgroup a row: 32 rows of 16384 tokens 25.3 | 22.3; of 32768 32 rows 25 | 31, 64 27 | 31, 72 38 | 31, 128 41 | 32, 256 67 | 32; of
// 65536 32 rows 29 | 56, 64 43 | 57, 96 57 | 58, 128 72 | 58; of 131072 64 rows 72 | 110, 72 86 | 113, 96 101 | 114, 128 129 | 115.  (So
// up to some hundred rows of 131072 would still be faster by segments; the rule does not go by length.)
constexpr int kFewKeptRows = 64;
constexpr int kWholeRow = 24576;

// Rows of a cache moved to where they stay, and the weights with them.
struct EvictArgs {
  const int32_t* kept;
  const int32_t* kept_lens;
  const int32_t* table;    // pages that the rows go to, or null: in place
  float* weights;
  int64_t seq_stride, weight_stride;
  int32_t heads, budget;
  int32_t table_pages;
  int32_t weight_units;    // workgroups of a sequence that move weights,
  int32_t units;           // and all of them: H * 2 * slices * splits more
  int32_t slices, splits;  // of a row's bytes; of the rows
  int32_t k_slices, v_slices, k_bytes, v_bytes;  // of a row
  int32_t piece_bytes, log2_lanes;               // a lane's part of a row, and the lanes of a slice
};

// Threads of a workgroup that moves rows to other pages, and in place (32 ragged sequences cut to 2048 tokens of 4 bits: 1024
// threads 39 us, 512 45, 256 57).
constexpr int kMoveThreads = 256;
constexpr int kChainThreads = 1024;
constexpr int kRowsAhead = 8;        // rows of a thread on their way at once
// Rows of a workgroup on their way at once, whose slices are so many lanes wide (narrow ones fewer than that, for their
// places are in LDS).
constexpr int move_rows(int threads, int log2_lanes) { return (threads * kRowsAhead) >> (log2_lanes < 2 ? 2 : log2_lanes); }

// Tokens of a sequence, and how many of them stay, from what the device's arrays hold.
constexpr int32_t kept_len(const ServeArgs& s, int32_t kv_len) {
  return kv_len < 0 ? 0 : kv_len < s.max_kv ? kv_len : s.max_kv;
}
constexpr int32_t kept_budget(const KeepArgs& a, int32_t n, int32_t budget) {
  budget = budget < 0 ? 0 : budget < a.budget ? budget : a.budget;
  return budget < n ? budget : n;
}

// Of few rows (up to few_tiles row tiles of 16 a sequence and KV head; 32 sequences of 8192 tokens, 8 heads of 128, 32 rows, as few |
// as many: 60 | 82 us in 4 bits, 104 | 153 in 16; 4 rows 42 | 99 and 101 | 169): tokens of a wave at a time; sequences whose tokens
// are shared evenly (every workgroup adds up their lengths), and by how many workgroups: as many as run at once of the smallest
// form (4 bits of 128 channels, one row tile: three to a compute unit; others have two).  32 ragged sequences of 255 thousand tokens,
// 512 | 768 | 1024 | 1536 shares: 4 bits 51 | 52 | 54 | 53 us, in two row tiles 66 | 85 | 75 | 85; 8 bits 65 | 80 | 72 | 78; 16 bits
// 114 | 130 | 116 | 120 (512 would do for all); chunks of 128, 256 and 512 tokens, 4 bits, 65, 60 and 68.
// With a window tokens are cut into chunks of up to kMostChunk that leave two to four thousand, where there are that many.
// Window 1024 and 4 sinks, chunks of 32 | 64 | 128 | 256 | 512: the same sequences 4 bits 87 | 53 | 41 | 39 | 44 us, 16 bits 103 | 65 |
// 53 | 51 | 69 (the rule: 256); one of 131072 42 | 26 | 22 | 21 | 33 (64).  Four of 700, window 256: 9.4 | 10.6 | 13.6 | 17 | 21 (32).
constexpr int kFewWaves = 4;
constexpr int kMostChunk = 512;
constexpr int kMostShared = 512;
constexpr int kShares = 768;
// Of many rows: tokens of a workgroup, rows of a tile, and its bytes (queries, and 5 numbers a row and 8 of all).
constexpr int weigh_tokens(int head_dim) { return head_dim > 128 ? 128 : 256; }
constexpr int kWeighRows = 32;
constexpr int weigh_tile_bytes(int head_dim) { return kWeighRows * (2 * head_dim + 20) + 32; }

// A launch has fewer than 2^32 threads: so many workgroups of 256, a quarter of them of 1024.
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
// (serve_args' part of the batch, without its page_table.)
pkv_status_t batch_args(const pkv_model_t* model, const pkv_batch_t* batch, bool pointers, ServeArgs* out);
pkv_status_t rotate_args(const pkv_model_t& m, const ServeArgs& s, const pkv_rotation_t* rotation, RotateArgs* out);
pkv_status_t attend_args(const ServeArgs& s, const pkv_attention_t* a, bool pointers, AttendArgs* out);
AttendLaunch attend_launch(const ServeArgs& s, const AttendArgs& a);
pkv_status_t weigh_args(const ServeArgs& s, const pkv_attention_t* a, const pkv_weights_t* w, bool pointers, WeighArgs* out,
                        WeighLaunch* launch);

pkv_status_t keep_args(const ServeArgs& s, const pkv_weights_t* w, const pkv_kept_t* k, bool pointers, KeepArgs* out,
                       uint64_t* workspace_bytes);
pkv_status_t evict_args(const ServeArgs& s, const pkv_kept_t* k, const pkv_weights_t* w, const int32_t* page_table,
                        int32_t table_pages, EvictArgs* out);

}  // namespace pkv

#endif  // PKV_SERVE_H
