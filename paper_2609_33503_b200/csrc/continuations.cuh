// Internal: what the calls over many continuations of a context share: argument checks, the per-context table, workspace, tensor maps.
#pragma once
#include "common.cuh"
#include <cuda.h>
#include <algorithm>

namespace relaxkv {

// Per-context values of a step over continuations, by value in the kernels' parameters.
struct ContTable {
  int n_req, n_seq;
  int seq_cu[kMaxReqInline + 1];
  int max_rows[kMaxReqInline];
  int ctx_len[kMaxReqInline];
  int blk_cu[kMaxReqInline + 1];       // prefix of the context blocks
  int tile_cu[kMaxReqInline + 1];      // call-specific prefix
  int pieces[kMaxReqInline];           // pieces (slots) that a context's keys are cut into
  long long tok_off[kMaxReqInline];
};

// Context of a sequence (in range).
__device__ __forceinline__ int context_of(const ContTable& ct, int seq) {
  int b = 0;
  for (int hi = ct.n_req; hi - b > 1;) { const int mid = (b + hi) >> 1; if (ct.seq_cu[mid] <= seq) b = mid; else hi = mid; }
  return b;
}

// Tokens of a context or of a sequence, at most: what a tile adds still fits 32 bits.
constexpr int kContTokensMost = 0x7fffff00;

inline bool block_size_ok(int32_t bs) { return bs == 16 || bs == 32 || bs == 64 || bs == 128; }

// check_shape, with contexts of no token
inline relaxkv_status check_contexts(const relaxkv_shape* s) {
  if (!s || !s->h_ctx_len) return RELAXKV_ERR_INVALID_ARG;
  if (s->n_req < 1 || s->n_q_heads < 1 || s->n_kv_heads < 1) return RELAXKV_ERR_INVALID_ARG;
  if (s->n_q_heads % s->n_kv_heads != 0) return RELAXKV_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (s->n_q_heads / s->n_kv_heads > 16 || s->n_req > kMaxReqInline) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  for (int b = 0; b < s->n_req; ++b) {
    if (s->h_ctx_len[b] < 0) return RELAXKV_ERR_INVALID_ARG;
    if (s->h_ctx_len[b] > kContTokensMost) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  }
  if (!(s->softmax_scale > 0.f)) return RELAXKV_ERR_INVALID_ARG;
  return RELAXKV_OK;
}

inline relaxkv_status check_store(const relaxkv_paged_cache* c, int32_t head_dim) {
  if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return RELAXKV_ERR_INVALID_ARG;
  if (!block_size_ok(c->block_size)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (c->n_blocks < 1 || (long long)c->n_blocks * c->block_size > 0x7fffffffLL) return RELAXKV_ERR_INVALID_ARG;     // slots are int32
  if (c->block_stride < head_dim || c->token_stride < head_dim || c->head_stride < head_dim) return RELAXKV_ERR_INVALID_ARG;
  if (c->block_stride % 8 || c->token_stride % 8 || c->head_stride % 8) return RELAXKV_ERR_INVALID_ARG;
  return RELAXKV_OK;
}

inline void fill_contexts(ContTable& t, const relaxkv_shape* s, const relaxkv_cache_view* c, int block_size) {
  t.n_req = s->n_req;
  t.n_seq = 0;
  t.seq_cu[0] = t.blk_cu[0] = t.tile_cu[0] = 0;
  for (int b = 0; b < s->n_req; ++b) {
    t.ctx_len[b] = s->h_ctx_len[b];
    t.tok_off[b] = c ? c->h_req_token_offset[b] : 0;
    t.blk_cu[b + 1] = t.blk_cu[b] + (block_size > 0 ? (int)(((long long)t.ctx_len[b] + block_size - 1) / block_size) : 0);
    t.seq_cu[b + 1] = t.max_rows[b] = t.tile_cu[b + 1] = t.pieces[b] = 0;
  }
}

// Checks the rows of a step and fills the table's sequences.  attend: row_len and, where max_len > 0, the tables are read, too.
inline relaxkv_status check_rows(const relaxkv_shape* s, const relaxkv_continuation_rows* r, bool attend, ContTable& t) {
  if (!r || !r->h_seq_cu || !r->h_max_rows || !r->row_cu || !r->row_seq) return RELAXKV_ERR_INVALID_ARG;
  if (r->n_seq < 1 || r->n_rows < 0 || r->h_seq_cu[0] != 0 || r->h_seq_cu[s->n_req] != r->n_seq) return RELAXKV_ERR_INVALID_ARG;
  if (r->n_rows > 0x7fffffffLL / (s->n_q_heads * 2)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (attend) {
    if (!r->row_len || r->max_len < 0) return RELAXKV_ERR_INVALID_ARG;
    if (r->max_len > kContTokensMost) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
    if (r->max_len > 0 && (!r->block_table || r->table_width < 1 || r->table_stride < r->table_width)) return RELAXKV_ERR_INVALID_ARG;
  }
  t.n_seq = r->n_seq;
  for (int b = 0; b < s->n_req; ++b) {
    if (r->h_seq_cu[b + 1] < r->h_seq_cu[b] || r->h_max_rows[b] < 0 || r->h_max_rows[b] > r->n_rows) return RELAXKV_ERR_INVALID_ARG;
    t.seq_cu[b + 1] = r->h_seq_cu[b + 1];
    t.max_rows[b] = r->h_max_rows[b];
  }
  return RELAXKV_OK;
}

// Scratch of the attention calls: partial results [slots][n_rows][H][D] and their log-sum-exps [slots][n_rows][H], one slot per piece that a
// row's keys are cut into.  Room for 4096 row-slots, and for four slots of every row.
constexpr int kContRowSlots = 4096, kContSlotsMost = 64;
inline int cont_slots(int64_t n_rows) {
  const int64_t by_room = kContRowSlots / std::max<int64_t>(1, n_rows);
  return (int)std::min<int64_t>(kContSlotsMost, std::max<int64_t>(4, by_room));
}
struct ContWs { size_t part_o, part_lse, scores, total; };
inline ContWs cont_ws(const relaxkv_shape* s, int64_t n_rows, int block_size) {
  ContWs w{};
  size_t a = 0;
  // (the most that this many rows or fewer can ask for)
  const size_t row_slots = (size_t)std::min<int64_t>(std::max<int64_t>(kContRowSlots, 4 * n_rows), kContSlotsMost * std::max<int64_t>(1, n_rows));
  w.part_o = a; a = align_up(a + row_slots * s->n_q_heads * s->head_dim * 4, 256);
  w.part_lse = a; a = align_up(a + row_slots * s->n_q_heads * 4, 256);
  w.total = a;
  if (block_size > 0) {
    long long most = 0;
    for (int b = 0; b < s->n_req; ++b) most = std::max(most, ((long long)s->h_ctx_len[b] + block_size - 1) / block_size);
    w.scores = 0;
    w.total = std::max(w.total, align_up((size_t)n_rows * s->n_kv_heads * most * 4, 256));
  }
  return w;
}

// K or V as [blocks, kv heads, D / 64, tokens, 64]: the box of one load is `box` tokens of one block and head, all dims, laid out in shared
// memory as D / 64 halves of box rows of 128 bytes, 128-byte swizzled.  A contiguous cache is one block of all its tokens.
bool make_block_map(CUtensorMap* m, const void* base, int D, uint64_t tokens, int n_kv_heads, uint64_t blocks, uint64_t token_stride,
                    uint64_t head_stride, uint64_t block_stride, uint32_t box);        // attention_sm100.cu

}  // namespace relaxkv
