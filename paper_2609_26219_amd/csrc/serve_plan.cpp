// Host half of the serving calls: argument checks and the choice of launches.
// Pure C++ (no HIP calls), so every check runs without a GPU.
#include <math.h>
#include <stddef.h>

#include <algorithm>

#include "serve.h"

namespace pkv {
namespace {

bool aligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

uint64_t head_bytes(const pkv_model_t& m, int tag) {
  return uint64_t(m.page_size) * m.head_dim * (kKeyBits[tag] + kValueBits[tag]) / 8;
}

int log2_of(int64_t x) {
  int r = 0;
  while ((int64_t(1) << r) < x) ++r;
  return r;
}

bool stride_ok(int64_t token, int64_t head, int32_t dim) {
  const int64_t most = int64_t(1) << 40;  // far from overflow with 2^31 rows' worth of offsets in bytes
  return token % 8 == 0 && head % 8 == 0 && head >= dim && token >= 0 && token <= most && head <= most;
}

}  // namespace

pkv_status_t batch_args(const pkv_model_t* model, const pkv_batch_t* batch, bool pointers, ServeArgs* out) {
  const pkv_status_t st = check_model(model);
  if (st != PKV_OK) return st;
  if (!batch) return PKV_ERR_INVALID_ARGUMENT;
  const pkv_model_t& m = *model;
  const pkv_batch_t& b = *batch;
  if (b.num_seqs >= kMostGroups || b.num_tokens >= kMostGroups) return PKV_ERR_INVALID_ARGUMENT;
  if (b.num_seqs < 0 || b.num_tokens < 0 || b.max_tokens < 0 || b.pages_per_seq < 1 || b.max_kv_len < 0)
    return PKV_ERR_INVALID_ARGUMENT;
  const int64_t reach = int64_t(b.pages_per_seq) * m.page_size;
  if (reach > (int64_t(1) << 30)) return PKV_ERR_INVALID_ARGUMENT;
  ServeArgs s{};
  s.token_start = b.token_start;
  s.kv_lens = b.kv_lens;
  s.positions = b.positions;
  s.page_table = b.page_table;
  s.num_seqs = b.num_seqs;
  s.num_tokens = b.num_tokens;
  s.max_tokens = b.max_tokens ? std::min(b.max_tokens, b.num_tokens) : b.num_tokens;
  s.pages_per_seq = b.pages_per_seq;
  s.max_kv = int32_t(b.max_kv_len ? std::min<int64_t>(b.max_kv_len, reach) : reach);
  s.pool_pages = m.pool_pages;
  s.log2P = log2_of(m.page_size);
  s.H = m.num_kv_heads;
  s.D = m.head_dim;
  s.bf16 = m.out_dtype == PKV_OUT_BF16;
  if (pointers && s.num_seqs > 0 && s.num_tokens > 0) {
    if (!b.token_start || !b.kv_lens) return PKV_ERR_INVALID_ARGUMENT;
    if (!aligned(b.token_start, 4) || !aligned(b.kv_lens, 4) || !aligned(b.positions, 4)) return PKV_ERR_INVALID_ARGUMENT;
  }
  *out = s;
  return PKV_OK;
}

pkv_status_t serve_args(const pkv_model_t* model, const pkv_paged_cache_t* cache, const pkv_batch_t* batch,
                        bool pointers, ServeArgs* out) {
  pkv_status_t st = check_model(model);
  if (st != PKV_OK) return st;
  if (!cache || !batch) return PKV_ERR_INVALID_ARGUMENT;
  const pkv_model_t& m = *model;
  if (cache->tag < PKV_TAG_FP16 || cache->tag > PKV_TAG_K4V4) return PKV_ERR_BAD_TAG;
  if (cache->layer < 0 || cache->layer >= m.num_layers) return PKV_ERR_INVALID_ARGUMENT;
  ServeArgs s{};
  st = batch_args(model, batch, pointers, &s);
  if (st != PKV_OK) return st;
  s.tag = cache->tag;
  if (s.tag == PKV_TAG_FP16) {
    s.page_stride = int64_t(m.page_size) * s.H * s.D * (m.kv_layout == PKV_KV_PAIRED ? 2 : 1);
  } else {
    s.head_stride = int64_t(head_bytes(m, s.tag));
    s.page_stride = s.head_stride * s.H;
    s.scale_stride = int64_t(s.H) * 2 * m.page_size;
    s.v_offset = int64_t(m.page_size) * s.D * kKeyBits[s.tag] / 8;
  }
  if (pointers) {
    if (s.num_seqs > 0 && s.num_tokens > 0 && (!s.page_table || !aligned(s.page_table, 4))) return PKV_ERR_INVALID_ARGUMENT;
    if (s.tag == PKV_TAG_FP16) {
      if (!cache->k_cache || !cache->v_cache || cache->cache_bytes < cache_bytes(m)) return PKV_ERR_INVALID_ARGUMENT;
      ByteRange ranges[2];
      int n = 0;
      if (!cache_ranges(m, cache->k_cache, cache->v_cache, cache_bytes(m), ranges, n)) return PKV_ERR_INVALID_ARGUMENT;
      const int64_t at = cache->layer * layer_elems(m);
      s.k_cache = static_cast<uint16_t*>(cache->k_cache) + at;
      s.v_cache = static_cast<uint16_t*>(cache->v_cache) + at;
    } else {
      uint64_t codes = 0, scales = 0;
      (void)pkv_cache_size(&m, s.tag, &codes, &scales);
      if (!cache->codes || !cache->scales || !aligned(cache->codes, 16) || !aligned(cache->scales, 16))
        return PKV_ERR_INVALID_ARGUMENT;
      if (cache->code_bytes < codes || cache->scale_bytes < scales) return PKV_ERR_INVALID_ARGUMENT;
      s.codes = static_cast<uint8_t*>(cache->codes) + cache->layer * m.pool_pages * s.page_stride;
      s.scales = static_cast<uint32_t*>(cache->scales) + cache->layer * m.pool_pages * s.scale_stride;
    }
  }
  *out = s;
  return PKV_OK;
}

pkv_status_t rotate_args(const pkv_model_t& m, const ServeArgs& s, const pkv_rotation_t* rotation, RotateArgs* out) {
  if (!rotation) return PKV_ERR_INVALID_ARGUMENT;
  const pkv_rotation_t& r = *rotation;
  if (r.num_heads < 0 || !isfinite(r.amplitude) || !aligned(r.position_offset, 4)) return PKV_ERR_INVALID_ARGUMENT;
  // (A workgroup counts a token's heads past the last by up to 2 * 128.)
  if (r.num_heads > (1 << 30) || int64_t(s.num_tokens) * r.num_heads >= (int64_t(1) << 31)) return PKV_ERR_INVALID_ARGUMENT;
  if (r.num_heads > 0) {
    if (!stride_ok(r.x_token_stride, r.x_head_stride, s.D) || !stride_ok(r.out_token_stride, r.out_head_stride, s.D))
      return PKV_ERR_INVALID_ARGUMENT;
    if (s.num_tokens > 0 && s.num_seqs > 0 && (!r.x || !r.out)) return PKV_ERR_INVALID_ARGUMENT;
    if (!aligned(r.x, 16) || !aligned(r.out, 16)) return PKV_ERR_INVALID_ARGUMENT;
    if (r.x == r.out && (r.x_token_stride != r.out_token_stride || r.x_head_stride != r.out_head_stride))
      return PKV_ERR_INVALID_ARGUMENT;
  }
  out->offset = r.position_offset;
  out->x = static_cast<const uint16_t*>(r.x);
  out->out = static_cast<uint16_t*>(r.out);
  out->x_token_stride = r.x_token_stride;
  out->x_head_stride = r.x_head_stride;
  out->out_token_stride = r.out_token_stride;
  out->out_head_stride = r.out_head_stride;
  out->amplitude = r.amplitude;
  out->heads = r.num_heads;
  out->rotary = rotary_dim(m);
  out->interleaved = m.rope_style == PKV_ROPE_INTERLEAVED;
  out->reserved = 0;
  for (int32_t j = 0; j < out->rotary / 2; ++j) out->freq[j] = rope_frequency(m, j);
  return PKV_OK;
}

pkv_status_t row_args(const ServeArgs& s, const void* k, const void* v, int64_t token_stride, int64_t head_stride,
                      RowArgs* out) {
  if (!stride_ok(token_stride, head_stride, s.D)) return PKV_ERR_INVALID_ARGUMENT;
  if (s.num_tokens > 0 && s.num_seqs > 0 && (!k || !v)) return PKV_ERR_INVALID_ARGUMENT;
  if (!aligned(k, 16) || !aligned(v, 16)) return PKV_ERR_INVALID_ARGUMENT;
  *out = RowArgs{static_cast<uint16_t*>(const_cast<void*>(k)), static_cast<uint16_t*>(const_cast<void*>(v)),
                 token_stride, head_stride};
  return PKV_OK;
}

pkv_status_t attend_args(const ServeArgs& s, const pkv_attention_t* a, bool pointers, AttendArgs* out) {
  if (!a) return PKV_ERR_INVALID_ARGUMENT;
  if (s.D != 64 && s.D != 128 && s.D != 256) return PKV_ERR_INVALID_ARGUMENT;
  if (a->num_q_heads < 1 || a->num_q_heads % s.H || a->window < 0 || a->sinks < 0) return PKV_ERR_INVALID_ARGUMENT;
  if (!(isfinite(a->scale) && a->scale > 0.0f)) return PKV_ERR_INVALID_ARGUMENT;
  if (int64_t(s.num_tokens) * a->num_q_heads >= (int64_t(1) << 31)) return PKV_ERR_INVALID_ARGUMENT;
  // The kernels multiply page numbers by 32-bit strides.
  const int64_t most = (int64_t(1) << 32) - 1;
  if (s.page_stride * (s.tag == PKV_TAG_FP16 ? 2 : 1) > most || s.scale_stride > most) return PKV_ERR_INVALID_ARGUMENT;
  AttendArgs r{};
  r.Hq = a->num_q_heads;
  r.group = r.Hq / s.H;
  r.window = a->window;
  r.sinks = a->sinks;
  r.scale = a->scale * 1.44269504088896340736f;
  if (pointers) {
    if (!stride_ok(a->q_token_stride, a->q_head_stride, s.D) || !stride_ok(a->out_token_stride, a->out_head_stride, s.D))
      return PKV_ERR_INVALID_ARGUMENT;
    if (s.num_tokens > 0 && s.num_seqs > 0 && (!a->q || !a->out)) return PKV_ERR_INVALID_ARGUMENT;
    if (!aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->lse, 4) || !aligned(a->workspace, 16))
      return PKV_ERR_INVALID_ARGUMENT;
    r.q = static_cast<const uint16_t*>(a->q);
    r.out = static_cast<uint16_t*>(a->out);
    r.lse = a->lse;
    r.q_token_stride = a->q_token_stride;
    r.q_head_stride = a->q_head_stride;
    r.out_token_stride = a->out_token_stride;
    r.out_head_stride = a->out_head_stride;
  }
  const AttendLaunch l = attend_launch(s, r);
  if (l.groups >= kMostGroups) return PKV_ERR_INVALID_ARGUMENT;
  if (l.workspace_bytes && int64_t(s.num_tokens) * r.Hq >= kMostGroups) return PKV_ERR_INVALID_ARGUMENT;
  r.tiles = l.tiles;
  r.row_tiles = l.row_tiles;
  r.splits = l.splits;
  r.pieces = l.pieces;
  r.part_rows = l.part_rows;
  r.chunk = l.chunk;
  if (pointers && l.workspace_bytes) {
    if (!a->workspace || a->workspace_bytes < l.workspace_bytes) return PKV_ERR_INVALID_ARGUMENT;
    r.part = static_cast<float*>(a->workspace);
    r.part_ml = reinterpret_cast<float*>(static_cast<char*>(a->workspace) + l.part_bytes);
  }
  *out = r;
  return PKV_OK;
}

AttendLaunch attend_launch(const ServeArgs& s, const AttendArgs& a) {
  AttendLaunch l{};
  if (s.num_seqs == 0 || s.num_tokens == 0) return l;  // no workgroups, no workspace
  const int64_t rows = int64_t(s.max_tokens) * a.group;
  const bool many = rows > few_shares(kKeyBits[s.tag]) * kRowTile * few_tiles(s.D);
  l.tiles = many ? many_tiles(s.D) : rows <= kRowTile ? 1 : few_tiles(s.D);
  l.row_tiles = int32_t((rows + kRowTile * l.tiles - 1) / (kRowTile * l.tiles));
  l.part_rows = int32_t(rows);
  const int64_t base = int64_t(s.num_seqs) * s.H * l.row_tiles;
  // tokens that a row tile may have to look at
  int64_t seen = s.max_kv;
  if (a.window > 0 && !s.positions) seen = std::min<int64_t>(seen, int64_t(a.sinks) + a.window + s.max_tokens);
  const int64_t tokens = many ? kManyElems / s.D : kTokenTile;
  const int64_t tiles = std::max<int64_t>(1, (seen + tokens - 1) / tokens + 1);
  uint64_t parts = 0;
  l.splits = 1;
  if (many) {
    // Workgroups for six times the compute units, of 16 tiles at least.  (1229 scattered rows of 32 heads: 578 us with
    // four times, 569 with six, 587 with eight; 2825 rows behind 10240 tokens: 598 with four and six, which leave them
    // uncut, 605 and 79 more to join with eight.)
    l.chunk = 16;
    l.splits = int32_t(std::max<int64_t>(1, std::min<int64_t>(6 * 256 / base, tiles / l.chunk)));
    l.groups = base * l.splits;
    if (l.splits > 1) parts = uint64_t(s.num_tokens) * a.Hq * l.splits;
  } else if (tiles <= (base >= 256 ? kWholeTilesOfMany : kWholeTiles)) {
    l.groups = base;
  } else {
    // As many workgroups as run at once, of two tiles a wave at least; where the sequences alone are more than half of
    // that, two rounds of them and half as many again as there are sequences.  (One tile a wave: 8 tokens behind 8192 take
    // 17.2 + 5.5 us instead of 14.2 + 4.6; four: one behind 1500 11.4 instead of 9.3.)
    const int64_t at_once = 256 * (s.D > 128 || l.tiles > 1 ? 2 : 3) / (int64_t(s.H) * l.row_tiles);
    l.chunk = 8;
    int64_t pieces = at_once;
    if (s.num_seqs > at_once / 2) pieces = std::max<int64_t>(2 * at_once, s.num_seqs + s.num_seqs / 2 + 1);
    pieces = std::min<int64_t>(pieces, s.num_seqs * ((tiles - 1) / l.chunk + 1) + 1);
    l.pieces = int32_t(std::max<int64_t>(pieces, s.num_seqs + 1));
    l.groups = int64_t(l.pieces) * s.H * l.row_tiles;
    parts = uint64_t(l.pieces) * s.H * l.part_rows;
  }
  l.part_bytes = parts * s.D * 4;
  l.workspace_bytes = l.part_bytes + parts * 8;
  return l;
}

namespace {

// The arrays of a call that goes over sequences, whether it has rows or not.
bool seqs_ok(const ServeArgs& s) {
  return s.token_start && s.kv_lens && s.page_table && aligned(s.token_start, 4) && aligned(s.kv_lens, 4) &&
         aligned(s.page_table, 4);
}

// Rows of numbers, one a token: whether they are laid out without overlap.
bool weights_ok(const ServeArgs& s, const pkv_weights_t& w) {
  const int64_t most = int64_t(1) << 40;
  if ((w.heads != 1 && w.heads != s.H) || w.tokens < s.max_kv || w.tokens > most) return false;
  if (w.heads > 1 && (w.head_stride < w.tokens || w.head_stride > most)) return false;
  const int64_t whole = (w.heads > 1 ? (w.heads - 1) * w.head_stride : 0) + w.tokens;
  return s.num_seqs <= 1 || (w.seq_stride >= whole && w.seq_stride <= most);
}

}  // namespace

pkv_status_t weigh_args(const ServeArgs& s, const pkv_attention_t* a, const pkv_weights_t* weights, bool pointers,
                        WeighArgs* out, WeighLaunch* launch) {
  if (!a || !weights) return PKV_ERR_INVALID_ARGUMENT;
  const pkv_weights_t& w = *weights;
  if (s.D != 64 && s.D != 128 && s.D != 256) return PKV_ERR_INVALID_ARGUMENT;
  if (a->num_q_heads < 1 || a->num_q_heads % s.H || a->window < 0 || a->sinks < 0) return PKV_ERR_INVALID_ARGUMENT;
  // (The rows' lse is divided by the scale.)
  if (!(isfinite(a->scale) && a->scale >= 0x1p-64f) || !isfinite(w.decay)) return PKV_ERR_INVALID_ARGUMENT;
  if (int64_t(s.num_tokens) * a->num_q_heads >= (int64_t(1) << 31)) return PKV_ERR_INVALID_ARGUMENT;
  // The kernels multiply page numbers by 32-bit strides.
  const int64_t most = (int64_t(1) << 32) - 1;
  if (s.page_stride * (s.tag == PKV_TAG_FP16 ? 2 : 1) > most || s.scale_stride > most) return PKV_ERR_INVALID_ARGUMENT;
  if (!weights_ok(s, w)) return PKV_ERR_INVALID_ARGUMENT;
  WeighArgs r{};
  r.Hq = a->num_q_heads;
  r.group = r.Hq / s.H;
  r.window = a->window;
  r.sinks = a->sinks;
  r.scale = a->scale * 1.44269504088896340736f;
  r.joint = w.heads == 1;
  r.decay = w.decay;
  r.seq_stride = w.seq_stride;
  r.head_stride = w.heads > 1 ? w.head_stride : 0;

  WeighLaunch l{};
  l.splits = l.subs = 1;
  if (s.num_seqs > 0) {
    const int64_t rows = int64_t(s.max_tokens) * r.group;
    if (rows <= kRowTile * few_tiles(s.D)) {
      l.few_tiles = rows <= kRowTile ? 1 : 2;
      // A workgroup's waves take a KV head each, or parts of the tokens where there are fewer.
      while (l.subs < kFewWaves && l.subs * 2 * s.H <= kFewWaves) l.subs *= 2;
      if (r.window == 0 && s.num_seqs <= kMostShared) {
        l.groups = std::max<int64_t>(1, std::min<int64_t>(kShares, (int64_t(s.num_seqs) * s.max_kv - 1) / (kTokenTile * l.subs) + 1));
      } else {
        l.chunk = kTokenTile * l.subs;
        while (l.chunk < kMostChunk && int64_t(s.num_seqs) * s.max_kv / l.chunk >= 4096) l.chunk *= 2;
        l.tiles = int32_t((int64_t(s.max_kv) + l.chunk - 1) / l.chunk);
        l.groups = int64_t(s.num_seqs) * l.tiles;
      }
    } else {
      const int tokens = weigh_tokens(s.D);
      l.tiles = int32_t((int64_t(s.max_kv) + tokens - 1) / tokens);
      const int64_t base = int64_t(s.num_seqs) * l.tiles * s.H;
      // Workgroups for 24 times the compute units, of 32 row tiles at least.  (8192 rows of 32 heads over 8192 tokens: 375 us
      // with six times, 365 with twelve, 358 with 24.)
      l.splits = int32_t(std::max<int64_t>(1, std::min<int64_t>(24 * 256 / base, rows / 1024)));
      l.groups = base * l.splits;
      if (l.splits > 1 || (r.joint && s.H > 1)) {
        l.part_bytes = (uint64_t(l.splits) * s.H * s.num_seqs * s.max_kv * 4 + 15) / 16 * 16;
        l.join_groups = int64_t(s.num_seqs) * w.heads * ((int64_t(s.max_kv) + 255) / 256);
      }
      l.row_tiles = int32_t((rows + kWeighRows - 1) / kWeighRows);
      l.all_tiles = int64_t(s.num_tokens) * r.group / kWeighRows + s.num_seqs + 1;
      l.prepare_groups = int64_t(s.num_seqs) * l.row_tiles * s.H;
      l.workspace_bytes = l.part_bytes + uint64_t(l.all_tiles) * s.H * weigh_tile_bytes(s.D);
    }
    if (l.groups >= kMostGroups || l.join_groups >= kMostGroups || l.prepare_groups >= kMostGroups)
      return PKV_ERR_INVALID_ARGUMENT;
  }
  r.tiles = l.tiles;
  r.chunk = l.chunk;
  r.subs = l.subs;
  r.splits = l.splits;
  r.row_tiles = l.row_tiles;
  r.all_tiles = l.all_tiles;
  if (pointers) {
    if (!stride_ok(a->q_token_stride, a->q_head_stride, s.D)) return PKV_ERR_INVALID_ARGUMENT;
    if (s.num_seqs > 0) {  // (a call without rows still lets the weights fade)
      if (!seqs_ok(s) || !w.out || (w.decay != 0.0f && !w.weights)) return PKV_ERR_INVALID_ARGUMENT;
      if (s.num_tokens > 0 && (!a->q || !a->lse)) return PKV_ERR_INVALID_ARGUMENT;
    }
    if (!aligned(a->q, 16) || !aligned(a->lse, 4) || !aligned(w.weights, 4) || !aligned(w.out, 4) ||
        !aligned(a->workspace, 16))
      return PKV_ERR_INVALID_ARGUMENT;
    if (l.workspace_bytes && (!a->workspace || a->workspace_bytes < l.workspace_bytes)) return PKV_ERR_INVALID_ARGUMENT;
    r.q = static_cast<const uint16_t*>(a->q);
    r.q_token_stride = a->q_token_stride;
    r.q_head_stride = a->q_head_stride;
    r.lse = a->lse;
    r.weights = w.decay != 0.0f ? w.weights : nullptr;
    r.out = w.out;
    r.part = l.part_bytes ? static_cast<float*>(a->workspace) : nullptr;
    r.rows = l.workspace_bytes ? static_cast<char*>(a->workspace) + l.part_bytes : nullptr;
  }
  *out = r;
  *launch = l;
  return PKV_OK;
}

namespace {

pkv_status_t kept_ok(const ServeArgs& s, const pkv_kept_t* k, const pkv_weights_t* w, bool pointers) {
  if (!k || (k->heads != 1 && k->heads != s.H)) return PKV_ERR_INVALID_ARGUMENT;
  if (k->budget < 0 || k->budget > (1 << 30) || k->sinks < 0 || k->recent < 0) return PKV_ERR_INVALID_ARGUMENT;
  if (w && (!weights_ok(s, *w) || w->heads != k->heads)) return PKV_ERR_INVALID_ARGUMENT;
  if (int64_t(s.num_seqs) * k->heads >= kMostGroups / 4) return PKV_ERR_INVALID_ARGUMENT;  // (of 1024 threads)
  if (!pointers) return PKV_OK;
  if (!aligned(k->kept, 4) || !aligned(k->kept_lens, 4) || !aligned(k->budgets, 4) || !aligned(s.kv_lens, 4))
    return PKV_ERR_INVALID_ARGUMENT;
  if (s.num_seqs > 0 && (!s.kv_lens || !k->kept_lens || (k->budget > 0 && !k->kept))) return PKV_ERR_INVALID_ARGUMENT;
  return PKV_OK;
}

}  // namespace

pkv_status_t keep_args(const ServeArgs& s, const pkv_weights_t* w, const pkv_kept_t* k, bool pointers, KeepArgs* out,
                       uint64_t* workspace_bytes) {
  if (!w) return PKV_ERR_INVALID_ARGUMENT;
  const pkv_status_t st = kept_ok(s, k, w, pointers);
  if (st != PKV_OK) return st;
  if (pointers && (!aligned(w->weights, 4) || (s.num_seqs > 0 && !w->weights))) return PKV_ERR_INVALID_ARGUMENT;
  // Workgroups read lengths and budgets while others write kept_lens.
  auto apart = [&](const int32_t* p, const int32_t* q) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
    return (x < y ? y - x : x - y) >= uintptr_t(s.num_seqs) * 4;
  };
  if (pointers && s.num_seqs > 0 &&
      (!apart(k->kept_lens, s.kv_lens) || (k->budgets && !apart(k->kept_lens, k->budgets))))
    return PKV_ERR_INVALID_ARGUMENT;
  KeepArgs a{};
  a.weights = w->weights;
  a.budgets = k->budgets;
  a.kept = k->kept;
  a.kept_lens = k->kept_lens;
  a.seq_stride = w->seq_stride;
  a.head_stride = w->heads > 1 ? w->head_stride : 0;
  a.heads = k->heads;
  a.budget = k->budget;
  a.sinks = k->sinks;
  a.recent = k->recent;
  const int64_t rows = int64_t(s.num_seqs) * k->heads;
  uint64_t counts = 0, lists = 0, segment = 0;
  if (rows > 0 && rows <= kFewKeptRows && s.max_kv > kWholeRow) {
    a.segments = (s.max_kv + kKeepSegment - 1) / kKeepSegment;
    const uint64_t all = uint64_t(rows) * a.segments;
    counts = all * 2048 * 4;
    lists = all * kKeepSegment * 4;
    segment = (all * sizeof(KeepSegment) + 15) / 16 * 16;
    if (int64_t(all) >= kMostGroups / 4) return PKV_ERR_INVALID_ARGUMENT;
  }
  *workspace_bytes = a.segments ? counts + lists + segment + uint64_t(rows) * sizeof(KeepRow) : 0;
  if (pointers && a.segments) {
    if (!k->workspace || !aligned(k->workspace, 16) || k->workspace_bytes < *workspace_bytes) return PKV_ERR_INVALID_ARGUMENT;
    char* at = static_cast<char*>(k->workspace);
    a.counts = reinterpret_cast<uint32_t*>(at);
    a.lists = reinterpret_cast<uint32_t*>(at + counts);
    a.segment = reinterpret_cast<KeepSegment*>(at + counts + lists);
    a.row = reinterpret_cast<KeepRow*>(at + counts + lists + segment);
  }
  *out = a;
  return PKV_OK;
}

pkv_status_t evict_args(const ServeArgs& s, const pkv_kept_t* k, const pkv_weights_t* w, const int32_t* page_table,
                        int32_t table_pages, EvictArgs* out) {
  const pkv_status_t st = kept_ok(s, k, w, true);
  if (st != PKV_OK) return st;
  if (!aligned(page_table, 4) || (page_table && table_pages < 1)) return PKV_ERR_INVALID_ARGUMENT;
  if (page_table && page_table == s.page_table && table_pages != s.pages_per_seq) return PKV_ERR_INVALID_ARGUMENT;
  if (w && (!aligned(w->out, 4) || (s.num_seqs > 0 && !w->out))) return PKV_ERR_INVALID_ARGUMENT;
  if (s.num_seqs > 0 && (!s.page_table || !aligned(s.page_table, 4))) return PKV_ERR_INVALID_ARGUMENT;
  EvictArgs e{};
  e.kept = k->kept;
  e.kept_lens = k->kept_lens;
  e.table = page_table == s.page_table ? nullptr : page_table;  // the batch's own pages are in place
  e.table_pages = table_pages;
  e.heads = k->heads;
  e.budget = k->budget;
  if (w) {
    e.weights = w->out;
    e.seq_stride = w->seq_stride;
    e.weight_stride = w->heads > 1 ? w->head_stride : 0;
    e.weight_units = w->heads;
  }
  e.k_bytes = s.D * kKeyBits[s.tag] / 8;
  e.v_bytes = s.D * kValueBits[s.tag] / 8;
  e.piece_bytes = e.k_bytes % 16 || e.v_bytes % 16 ? 8 : 16;
  // Slices: whole rows (up to 256 bytes) to other pages (85547 tokens of 16-bit rows cut to 14000: 39 us, in slices of 64 bytes
  // 68); in place as wide as leaves a compute unit its workgroup, 64 bytes at least.
  const int32_t pieces = std::max(e.k_bytes, e.v_bytes) / e.piece_bytes;
  while (e.log2_lanes < 4 && (1 << e.log2_lanes) < pieces) ++e.log2_lanes;
  auto slices_of = [&](int32_t bytes) {
    return (bytes / e.piece_bytes + (1 << e.log2_lanes) - 1) >> e.log2_lanes;
  };
  while (!e.table && e.log2_lanes > 2 &&
         int64_t(s.num_seqs) * s.H * (slices_of(e.k_bytes) + slices_of(e.v_bytes)) < 256)
    --e.log2_lanes;
  e.k_slices = slices_of(e.k_bytes);
  e.v_slices = slices_of(e.v_bytes);
  e.slices = std::max(e.k_slices, e.v_slices);
  const int64_t chunk = move_rows(kMoveThreads, e.log2_lanes);
  e.splits = 1;
  if (e.table) e.splits = int32_t(std::max<int64_t>(1, (std::min<int64_t>(e.budget, s.max_kv) + chunk - 1) / chunk));
  const int64_t units = e.weight_units + int64_t(s.H) * 2 * e.slices * e.splits;
  if (units * std::max(1, s.num_seqs) >= (e.table ? kMostGroups : kMostGroups / (kChainThreads / 256)))
    return PKV_ERR_INVALID_ARGUMENT;
  e.units = int32_t(units);
  *out = e;
  return PKV_OK;
}

}  // namespace pkv

extern "C" {

pkv_status_t pkv_cache_size(const pkv_model_t* model, int32_t tag, uint64_t* code_bytes, uint64_t* scale_bytes) {
  const pkv_status_t st = pkv::check_model(model);
  if (st != PKV_OK) return st;
  if (tag < PKV_TAG_FP16 || tag > PKV_TAG_K4V4) return PKV_ERR_BAD_TAG;
  if (!code_bytes || !scale_bytes) return PKV_ERR_INVALID_ARGUMENT;
  const uint64_t heads = tag == PKV_TAG_FP16 ? 0 : uint64_t(model->num_layers) * model->pool_pages * model->num_kv_heads;
  *code_bytes = heads * pkv::head_bytes(*model, tag);
  *scale_bytes = heads * 2 * model->page_size * 4;
  return PKV_OK;
}

pkv_status_t pkv_attention_workspace(const pkv_model_t* model, const pkv_paged_cache_t* cache, const pkv_batch_t* batch,
                                     const pkv_attention_t* attention, uint64_t* bytes) {
  if (!bytes) return PKV_ERR_INVALID_ARGUMENT;
  pkv::ServeArgs s;
  pkv::AttendArgs a;
  pkv_status_t st = pkv::serve_args(model, cache, batch, false, &s);
  if (st == PKV_OK) st = pkv::attend_args(s, attention, false, &a);
  if (st != PKV_OK) return st;
  *bytes = pkv::attend_launch(s, a).workspace_bytes;
  return PKV_OK;
}

pkv_status_t pkv_attention_weights_workspace(const pkv_model_t* model, const pkv_paged_cache_t* cache,
                                             const pkv_batch_t* batch, const pkv_attention_t* attention,
                                             const pkv_weights_t* weights, uint64_t* bytes) {
  if (!bytes) return PKV_ERR_INVALID_ARGUMENT;
  pkv::ServeArgs s;
  pkv::WeighArgs a;
  pkv::WeighLaunch l;
  pkv_status_t st = pkv::serve_args(model, cache, batch, false, &s);
  if (st == PKV_OK) st = pkv::weigh_args(s, attention, weights, false, &a, &l);
  if (st != PKV_OK) return st;
  *bytes = l.workspace_bytes;
  return PKV_OK;
}

pkv_status_t pkv_cache_keep_workspace(const pkv_model_t* model, const pkv_batch_t* batch, const pkv_weights_t* weights,
                                      const pkv_kept_t* kept, uint64_t* bytes) {
  if (!bytes) return PKV_ERR_INVALID_ARGUMENT;
  pkv::ServeArgs s;
  pkv::KeepArgs a;
  pkv_status_t st = pkv::batch_args(model, batch, false, &s);
  if (st == PKV_OK) st = pkv::keep_args(s, weights, kept, false, &a, bytes);
  return st;
}

}  // extern "C"
