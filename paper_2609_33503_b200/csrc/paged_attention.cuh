// Internal: the streaming attention over listed context blocks and paged tokens, and the merge of partial results.
#pragma once
#include "continuations.cuh"
#include "sm100_ptx.cuh"

namespace relaxkv {

// What a row's keys are made of besides its own tokens.
enum ContextKeys { CTX_KEYS_NONE = 0, CTX_KEYS_LISTED = 1, CTX_KEYS_ALL = 2 };

constexpr int kPagCluster = 8;         // blocks of a cluster, at most

struct PagedAttnArgs {
  const uint16_t* q;
  uint16_t* out;
  float *lse_out, *part_o, *part_lse;
  const int *row_seq, *row_len, *row_cu, *table, *lists;
  long long table_stride, n_rows;
  int table_width, max_len, n_select, n_blocks;
  int listed_most;                     // entries of a list that are blocks, at most
  int H, Hkv, n_seq;
  int ctx_keys;                        // ContextKeys
  int ctx_block, page;                 // tokens of a context block and of a block of the store
  int n_splits;                        // pieces a row's keys are cut into
  int cluster;                         // 1: a row's pieces are a cluster of blocks, which merges them and what the prefix kernel has left
  int behind_prefix;                   // 1: launched by the prefix kernel, once the kernels in front of that one are complete
  // clusters: a block's units of 32 threads' worth of results, units at once, groups of warps that share one, and every warp's group (4 bits each)
  int merge_units, merge_across, merge_groups;
  uint32_t merge_group_of;
  int slot0, n_slots;                  // first slot of these pieces, slots in all; one in all: results go to out
  float scale_log2;
};

// A row's sequence (-1: not one to work on), its own tokens and its context.
struct RowCheck { int seq, len, ctx; };

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int token, int head, int block) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(0), "r"(token), "r"(0), "r"(head), "r"(block) : "memory");
}

// Requests a box into L2 (nothing is written to this SM).
__device__ __forceinline__ void tma_prefetch_5d(const CUtensorMap* m, int token, int head, int block) {
  asm volatile("cp.async.bulk.prefetch.tensor.5d.L2.global.tile [%0, {%1, %2, %3, %4, %5}];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(0), "r"(token), "r"(0), "r"(head), "r"(block) : "memory");
}

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// tell: the reason why a row is left out is reported.
__device__ __forceinline__ RowCheck known_row(const PagedAttnArgs& a, const ContTable& ct, long long row, bool tell, DeviceStatus* st) {
  RowCheck r = {a.row_seq[row], a.row_len[row], 0};
  if (r.seq == -1) return r;
  const bool known = r.seq >= 0 && r.seq < a.n_seq;
  if (!known || r.len < 0 || r.len > a.max_len || (a.max_len > 0 && r.len > (long long)a.table_width * a.page)) {
    if (tell) report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_ATTN, known ? r.len : r.seq, (int)row);
    r.seq = -1;
    return r;
  }
  r.ctx = context_of(ct, r.seq);
  return r;
}
// Whether the rows [first, end) of a context are what the host's bounds and the step's rows allow, and this row is one of them.
__device__ __forceinline__ bool rows_fit(const PagedAttnArgs& a, const ContTable& ct, int ctx, int first, int end, long long row) {
  return first >= 0 && end <= a.n_rows && end - first <= ct.max_rows[ctx] && row >= first && row < end;
}
__device__ __forceinline__ RowCheck check_row(const PagedAttnArgs& a, const ContTable& ct, long long row, bool tell, DeviceStatus* st) {
  RowCheck r = known_row(a, ct, row, tell, st);
  if (r.seq < 0) return r;
  const int first = a.row_cu[ct.seq_cu[r.ctx]], end = a.row_cu[ct.seq_cu[r.ctx + 1]];
  if (!rows_fit(a, ct, r.ctx, first, end, row)) {
    if (tell) report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_ATTN, end - first, r.ctx);
    r.seq = -1;
  }
  return r;
}

// The largest cluster of at most n blocks of which `items` run at once (of blocks of four consumer warps).  Clusters live within a GPC, so they fill the
// GPU less than their blocks by themselves: 72 clusters of four are one more than fit, and took twice as long as 71.
int cluster_that_fits(const relaxkv_shape* shape, int n, long long items);

relaxkv_status launch_paged_attention(const relaxkv_shape* shape, const relaxkv_cache_view* cache, const relaxkv_paged_cache* store,
                                      const ContTable& ct, PagedAttnArgs a, cudaStream_t stream);
// out = sum over the slots of w_s O_s / sum w_s, w_s = exp(lse_s - max)
relaxkv_status launch_continuation_merge(const ContTable& ct, const PagedAttnArgs& a, int D, cudaStream_t stream);

}  // namespace relaxkv
