// Attention of single rows over listed blocks of their context and over their own tokens in the paged store
// (relaxkv_block_sparse_attention, and the own tokens of relaxkv_shared_prefix_attention).
//
// Every key and value meets the G <= 16 query heads of one KV head once: bound by the bytes of K and V.  A block of the launch owns (row, KV
// head, piece of the row's keys); a producer warp streams 64-key tiles through a ring in shared memory, one TMA box per block of the cache (its
// lanes look the block numbers up a tile ahead and each issues its own box, K and V), and four consumer warps take 16 keys of a tile each:
// S = Q K^T and O += P V as warp-level MMAs whose 16 rows are the heads (a 128-row tcgen05 tile would be 3 to 6 % full), softmax on the
// fragments (weights are rounded to bf16 for the product with V, their sums are of the unrounded ones in fp32).  16 keys never straddle a block, so a chunk's valid keys are one number.  Tiles of 64 keys and three stages leave room for two
// blocks per SM, which hide each other's starts; many rows of few keys go to blocks of two consumer warps or one, with tiles as much smaller (the
// rule and its figures: continuation_splits.cuh).
// A row's pieces merge among themselves where a cluster of up to eight blocks is enough (four rows of 32 K, 64 blocks each: 15.9 us, 18.1 with a merge
// behind), and with what the prefix kernel has left of the row's context.
// Measured, 128 of 2048 blocks for each of 16 rows 66 us (5.9 TB/s of HBM; rows share blocks in L2); own tokens of 64 rows of 40 / 8 heads, 512 on
// average (131 MB), 33 us: a block's chain row -> block number -> first tile takes 3.4 us and its results 1, between them it has its tiles at the rate
// of HBM, and blocks of 1 to 17 tiles do not end together.  Whole passes of those two when they took 94 and 83.8: two stages and three blocks per SM
// 112 and 86.6, 32-key tiles and four blocks 136 / 86.9, 128-key tiles and one 102 / 86.4.  Resident blocks that walk several items, with the
// producer running ahead (a fixed share of items; items by cluster launch control; an equal share of tiles, found by a sum over the lengths) hid
// the chain but not the tail, or lost the rows' shared blocks in L2: the first kernel 72 / 71 / 80 us of the 66, the second 33 / 37 / 33.
// Every wait is bounded.
#include "paged_attention.cuh"
#include "continuation_splits.cuh"
#include "sm100_ptx.cuh"
#include <atomic>

namespace relaxkv {

using namespace ptx;

constexpr int kPagStages = 3;
constexpr float kLog2eP = 1.4426950408889634f, kLn2P = 0.6931471805599453f;

// WARPS: consumer warps, sixteen keys of a tile each.
template <int D, int WARPS>
struct PagSmem {
  static constexpr int kThreads = (WARPS + 1) * 32;
  static constexpr int kTile = 16 * WARPS;                        // keys per tile
  static constexpr int kEntries = WARPS;                          // boxes of a tile, at most
  static constexpr int kBlocksPerSm = WARPS == 4 ? 2 : WARPS == 2 ? 4 : 6;
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kStageBytes = 2 * kTileBytes;              // K tile | V tile
  static constexpr int kBar = kPagStages * kStageBytes;           // full[stages], empty[stages]
  static constexpr int kValid = kBar + 16 * kPagStages;           // valid keys of each box of a stage
  static constexpr int kMisc = kValid + 4 * kPagStages * kEntries;
  static constexpr int kTotal = kMisc + 16;
  static constexpr int kDynamic = kTotal + 1024;
};

__device__ __forceinline__ void ldsm_x4(uint32_t* r, uint32_t smem_addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t* r, uint32_t smem_addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(smem_addr) : "memory");
}
__device__ __forceinline__ void mma_16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// GMAX: heads of a KV head's group, at most (8 or 16).
template <int D, int GMAX, int WARPS>
__global__ void __launch_bounds__(PagSmem<D, WARPS>::kThreads, PagSmem<D, WARPS>::kBlocksPerSm)
paged_attention_kernel(const __grid_constant__ CUtensorMap tm_ck, const __grid_constant__ CUtensorMap tm_cv,
                       const __grid_constant__ CUtensorMap tm_pk, const __grid_constant__ CUtensorMap tm_pv,
                       const __grid_constant__ ContTable ct, const __grid_constant__ PagedAttnArgs a, DeviceStatus* st) {
  using L = PagSmem<D, WARPS>;
  constexpr int kThreads = L::kThreads, kTile = L::kTile, kEntries = L::kEntries;
  constexpr int kRowsUsed = GMAX > 8 ? 2 : 1;          // fragment rows gid (and gid + 8) that hold heads
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar_full = base + L::kBar, bar_empty = bar_full + 8 * kPagStages;
  volatile int* valid_s = reinterpret_cast<volatile int*>(base_ptr + L::kValid);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + L::kMisc);
  __shared__ float m_s[WARPS][GMAX], z_s[WARPS][GMAX];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.H / a.Hkv;
  // KV heads fastest; with clusters, whose blocks stand side by side, the pieces
  const int unit = a.cluster ? (int)blockIdx.x / a.n_splits : 0;
  const int hd = (int)((a.cluster ? unit : blockIdx.x) % a.Hkv), split = (int)(a.cluster ? blockIdx.x - unit * a.n_splits : blockIdx.x / a.Hkv % a.n_splits);
  const long long row = blockIdx.x / (a.Hkv * a.n_splits);
  if (threadIdx.x == 0) {
    for (int s = 0; s < kPagStages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, WARPS); }
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (threadIdx.x == WARPS * 32) {                  // (of maps that there are)
    if (a.ctx_keys != CTX_KEYS_NONE) { prefetch_tensormap(&tm_ck); prefetch_tensormap(&tm_cv); }
    if (a.max_len > 0) { prefetch_tensormap(&tm_pk); prefetch_tensormap(&tm_pv); }
  }
  // what the chain row -> block numbers -> keys begins with, into L2 while the kernels in front finish (prefetches only)
  if (warp == 0) {
    if (lane == 0) { prefetch_l2(a.row_seq + row); prefetch_l2(a.row_len + row); prefetch_l2(st); }
    if (lane < G) prefetch_l2(a.q + (row * a.H + hd * G + lane) * D);
    if (a.ctx_keys == CTX_KEYS_LISTED && lane * 32 < a.n_select) prefetch_l2(a.lists + (row * a.Hkv + hd) * a.n_select + lane * 32);
  }
  __syncthreads();
  // q, the rows and the appended tokens come from the kernels before.  The prefix kernel lets this one start when it has waited for those
  // itself; its own results are waited for where the first is read (and nothing is written before).
  if (!a.behind_prefix) griddep_wait();
  const int status = *reinterpret_cast<volatile int*>(&st->status);
  const bool teller = threadIdx.x == 0 && split == 0 && hd == 0;
  const RowCheck rc = known_row(a, ct, row, teller, st);
  // (a block of a cluster stays to the end: the others read its shared memory)
  const bool live = rc.seq >= 0 && status != RELAXKV_ERR_TIMEOUT;
  if (!live && !a.cluster) {
    griddep_wait();                                     // (the kernels behind rely on it)
    return;
  }
  // looked at when the results are written: more rows than the host's bound
  const int rows_first = a.row_cu[ct.seq_cu[rc.ctx]], rows_end = a.row_cu[ct.seq_cu[rc.ctx + 1]];
  // ---- this piece's tiles: the row's are [listed context blocks | own tokens] ----
  const int ctx_box = min(a.ctx_block, kTile), page_box = min(a.page, kTile);
  const int ctx_sub = a.ctx_block / ctx_box, page_sub = a.page / page_box;             // boxes of a block
  const int ctx_per = kTile / ctx_box, page_per = kTile / page_box;              // boxes of a tile
  const int ctx_len = ct.ctx_len[rc.ctx], ctx_blocks = (int)(((long long)ctx_len + a.ctx_block - 1) / a.ctx_block);
  int listed = a.ctx_keys == CTX_KEYS_NONE || ctx_len == 0 ? 0 : a.ctx_keys == CTX_KEYS_ALL ? ctx_blocks : a.n_select;      // blocks
  if (live && listed > ctx_blocks) {                    // a list longer than its context ends with entries that are none: only up to the last one that is
    const int* list = a.lists + (row * a.Hkv + hd) * a.n_select;
    for (bool any = false; listed > 0 && !any;) {
      int id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) id[u] = listed > 32 * u + lane ? list[listed - 1 - 32 * u - lane] : -1;
#pragma unroll
      for (int u = 0; u < 4 && !any; ++u) {
        const uint32_t some = __ballot_sync(0xffffffffu, id[u] != -1);
        any = some != 0;
        listed -= any ? __ffs((int)some) - 1 : min(listed, 32);
      }
    }
  }
  const int n_ctx = (listed * ctx_sub + ctx_per - 1) / ctx_per;
  const int n_tiles = live ? n_ctx + (rc.len + kTile - 1) / kTile : 0;
  const int per = (n_tiles + a.n_splits - 1) / a.n_splits;
  const int t0 = min(n_tiles, split * per), t1 = min(n_tiles, t0 + per);

  float frag_m[2] = {-INFINITY, -INFINITY}, frag_z[2] = {0.f, 0.f}, frag_o[D / 8][4];
#pragma unroll
  for (int d = 0; d < D / 8; ++d) frag_o[d][0] = frag_o[d][1] = frag_o[d][2] = frag_o[d][3] = 0.f;
  if (warp == WARPS) {
    // ================= producer: one lane per box =================
    const int* list = a.ctx_keys == CTX_KEYS_LISTED ? a.lists + (row * a.Hkv + hd) * a.n_select : nullptr;
    auto block_number = [&](int t) -> int {             // of this lane's box of tile t; -1: none
      if (t >= t1) return -1;
      if (t < n_ctx) {
        const int u = t * ctx_per + lane;
        return lane < ctx_per && u < listed * ctx_sub ? (list ? list[u / ctx_sub] : u / ctx_sub) : -1;
      }
      const int u = (t - n_ctx) * page_per + lane;
      return lane < page_per && u * page_box < rc.len ? a.table[rc.seq * a.table_stride + u / page_sub] : -1;
    };
    int id = block_number(t0);
    for (int t = t0, it = 0; t < t1; ++t, ++it) {
      const int s = it % kPagStages;
      const int id_next = block_number(t + 1);          // on its way while the ring is full
      if (it >= kPagStages) {
        const bool ok = mbar_wait(bar_empty + 8 * s, (uint32_t)((it / kPagStages) - 1) & 1, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) break;
      }
      const bool of_ctx = t < n_ctx;
      const int box = of_ctx ? ctx_box : page_box;
      int valid = 0, token = 0, block = 0;
      if (lane < (of_ctx ? ctx_per : page_per)) {
        if (of_ctx) {
          const int off = (t * ctx_per + lane) % ctx_sub * box;
          if (id >= 0 && id < ctx_blocks) {
            valid = max(0, min(box, ctx_len - (id * a.ctx_block + off)));
            token = (int)(ct.tok_off[rc.ctx] + (long long)id * a.ctx_block + off);
          } else if (id != -1) report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_ATTN, id, ctx_blocks);
        } else {
          const int u = (t - n_ctx) * page_per + lane, left = rc.len - u * box;
          token = u % page_sub * box;
          if (left > 0) {
            if (id >= 0 && id < a.n_blocks) { valid = min(box, left); block = id; }
            else report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_ATTN, id, a.n_blocks);
          }
        }
        valid_s[s * kEntries + lane] = valid;
      }
      const int n_boxes = __popc(__ballot_sync(0xffffffffu, valid > 0));
      __syncwarp();                                     // the valid keys of all boxes are written
      if (lane == 0) mbar_expect_tx(bar_full + 8 * s, (uint32_t)(n_boxes * box * D * 4));
      __syncwarp();
      if (valid > 0) {
        const uint32_t dst = base + s * L::kStageBytes + lane * box * D * 2;
        tma_load_5d(dst, of_ctx ? &tm_ck : &tm_pk, bar_full + 8 * s, token, hd, block);
        tma_load_5d(dst + L::kTileBytes, of_ctx ? &tm_cv : &tm_pv, bar_full + 8 * s, token, hd, block);
      }
      id = id_next;
    }
  } else {
    // ================= consumers =================
    const int gid = lane >> 2, tig = lane & 3;                        // fragment coordinates: row gid (and gid + 8), column pair tig
    uint32_t qa[D / 16][4];                                           // the heads as A fragments, the bf16 pairs as stored (the scale goes on S)
    const uint16_t* q_head = a.q + (row * a.H + hd * G) * D + tig * 2;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        qa[ks][h2 * 2] = gid < G ? *reinterpret_cast<const uint32_t*>(q_head + gid * D + ks * 16 + h2 * 8) : 0u;
        qa[ks][h2 * 2 + 1] = (GMAX > 8 && gid + 8 < G) ? *reinterpret_cast<const uint32_t*>(q_head + (gid + 8) * D + ks * 16 + h2 * 8) : 0u;
      }
    }
    for (int t = t0, it = 0; t < t1; ++t, ++it) {
      const int s = it % kPagStages;
      bool ok = mbar_wait(bar_full + 8 * s, (uint32_t)(it / kPagStages) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      const int box = t < n_ctx ? ctx_box : page_box, entry = warp * 16 / box, off = warp * 16 - entry * box;
      const int n_here = min(16, valid_s[s * kEntries + entry] - off);                 // keys of this warp's chunk that count
      if (n_here > 0) {
        const uint32_t half = (uint32_t)box * 128, chunk = (uint32_t)(entry * box * D * 2 + off * 128);
        const uint32_t kt = base + s * L::kStageBytes + chunk, vt = kt + L::kTileBytes;
        if (n_here < 16) {
          // V rows behind the valid ones belong to nobody (they may hold NaN, and 0 x NaN = NaN on the tensor core): zero them
          uint8_t* vrows = base_ptr + s * L::kStageBytes + L::kTileBytes + chunk;
          for (int i = lane; i < (16 - n_here) * (D / 8); i += 32) {
            const int r = n_here + i / (D / 8), c16 = i % (D / 8);
            *reinterpret_cast<uint4*>(vrows + (c16 >> 3) * half + r * 128 + (((c16 & 7) ^ (r & 7)) << 4)) = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();                                   // (the stage's next copy comes through the other proxy)
          __syncwarp();
        }
        // ---- S = Q K^T: two 8-key column tiles ----
        float sacc[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          sacc[j][0] = sacc[j][1] = sacc[j][2] = sacc[j][3] = 0.f;
          const int r = j * 8 + (lane & 7);
#pragma unroll
          for (int q4 = 0; q4 < D / 32; ++q4) {
            const int c16 = 4 * q4 + (lane >> 3);
            uint32_t kb[4];
            ldsm_x4(kb, kt + (c16 >> 3) * half + r * 128 + (((c16 & 7) ^ (r & 7)) << 4));
            mma_16816(sacc[j], qa[2 * q4], kb[0], kb[1]);
            mma_16816(sacc[j], qa[2 * q4 + 1], kb[2], kb[3]);
          }
        }
        // ---- online softmax: this lane holds, of rows gid (and gid + 8), keys 8 j + 2 tig (+ 1) ----
        uint32_t pa[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int rr = 0; rr < kRowsUsed; ++rr) {
          float mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float v = j * 8 + tig * 2 + e < n_here ? sacc[j][2 * rr + e] * a.scale_log2 : -INFINITY;
              sacc[j][2 * rr + e] = v;
              mx = fmaxf(mx, v);
            }
          }
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          const float m_new = fmaxf(frag_m[rr], mx), m_ref = m_new == -INFINITY ? 0.f : m_new;      // (every logit so far may be -inf)
          const float alpha = fast_exp2(frag_m[rr] - m_ref);
          frag_m[rr] = m_new;
          float z = 0.f;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float p0 = fast_exp2(sacc[j][2 * rr] - m_ref), p1 = fast_exp2(sacc[j][2 * rr + 1] - m_ref);
            z += p0 + p1;
            const __nv_bfloat162 p01 = __floats2bfloat162_rn(p0, p1);
            pa[j * 2 + rr] = *reinterpret_cast<const uint32_t*>(&p01);
          }
          frag_z[rr] = frag_z[rr] * alpha + z;                        // this lane's keys; the quad is added up at the end
#pragma unroll
          for (int d = 0; d < D / 8; ++d) { frag_o[d][2 * rr] *= alpha; frag_o[d][2 * rr + 1] *= alpha; }
        }
        // ---- O += P V: V fragments transposed out of the tile, two 8-dim column tiles per load ----
        const int r = ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
        for (int dp = 0; dp < D / 16; ++dp) {
          const int c16 = 2 * dp + (lane >> 4);
          uint32_t vb[4];
          ldsm_x4_trans(vb, vt + (c16 >> 3) * half + r * 128 + (((c16 & 7) ^ (r & 7)) << 4));
          mma_16816(frag_o[2 * dp], pa, vb[0], vb[1]);
          mma_16816(frag_o[2 * dp + 1], pa, vb[2], vb[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty + 8 * s);                  // this warp is through with the stage
    }
#pragma unroll
    for (int rr = 0; rr < kRowsUsed; ++rr) {
      frag_z[rr] += __shfl_xor_sync(0xffffffffu, frag_z[rr], 1);
      frag_z[rr] += __shfl_xor_sync(0xffffffffu, frag_z[rr], 2);
    }
  }
  __syncthreads();                                                    // every tile consumed: the ring is free
  griddep_launch();                                                   // (called first thing, sixteen rows of 16 K took 30.1 us, 29.4 so)
  // ---- the warps' results, added up in a fixed order: every warp adds up a quarter of the dims, the others' come through the ring's place
  // in fragment order (written head by head, a warp's stores met in eight banks and this took 1.3 us) ----
  constexpr int kOwn = D / 8 / WARPS;                             // of the 8-dim column tiles of O
  static_assert(WARPS * (WARPS - 1) * kOwn * 32 * kRowsUsed * 8 <= L::kBar, "they fit the ring");
  auto part_s = [&](int owner, int from, int i) -> float2* {          // warp `from`'s fragment of tile i of `owner`: this lane's place
    return reinterpret_cast<float2*>(base_ptr) + (((owner * (WARPS - 1) + from - (from > owner ? 1 : 0)) * kOwn + i) * 32 + lane) * kRowsUsed;
  };
  const int gid = lane >> 2, tig = lane & 3;
  float own[kOwn][2 * kRowsUsed];
  if (warp < WARPS && !*abort_flag) {
#pragma unroll
    for (int d = 0; d < D / 8; ++d) {
      if (d / kOwn == warp) {
#pragma unroll
        for (int e = 0; e < 2 * kRowsUsed; ++e) own[d % kOwn][e] = frag_o[d][e];
      } else {
#pragma unroll
        for (int rr = 0; rr < kRowsUsed; ++rr) part_s(d / kOwn, warp, d % kOwn)[rr] = make_float2(frag_o[d][2 * rr], frag_o[d][2 * rr + 1]);
      }
    }
#pragma unroll
    for (int rr = 0; rr < kRowsUsed; ++rr)
      if (tig == 0 && gid + 8 * rr < G) { m_s[warp][gid + 8 * rr] = frag_m[rr]; z_s[warp][gid + 8 * rr] = frag_z[rr]; }
  }
  __syncthreads();
  griddep_wait();
  const bool gave_up = *reinterpret_cast<volatile int*>(&st->status) == RELAXKV_ERR_TIMEOUT;      // the prefix kernel may have, meanwhile
  const bool aborted = *abort_flag != 0;
  if (aborted) {
    if (threadIdx.x == 0) report(st, RELAXKV_ERR_TIMEOUT, KID_PAGED_ATTN, (int)row, hd);
    const uint64_t tw = global_timer_ns();                            // copies still in flight: let them land
    while (global_timer_ns() - tw < 200000ull) __nanosleep(1000);
    if (!a.cluster) return;
  }
  const bool fits = rows_fit(a, ct, rc.ctx, rows_first, rows_end, row);
  if (live && !fits && teller) report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_ATTN, rows_end - rows_first, rc.ctx);
  if (!a.cluster && (gave_up || !fits)) return;
  // where a cluster's blocks find each other's results: [G][D] normalised, behind them the log-sum-exps (in log2 units; NaN: given up)
  constexpr int kResult = L::kBar / 2, kResultLse = kResult + GMAX * D * 4;
  static_assert(WARPS * (WARPS - 1) * kOwn * 32 * kRowsUsed * 8 <= kResult && kResultLse + GMAX * 4 <= L::kBar, "side by side in the ring");
  if (warp < WARPS) {
#pragma unroll
    for (int rr = 0; rr < kRowsUsed; ++rr) {
      const int g = gid + 8 * rr;
      if (g >= G) continue;
      float mb = -INFINITY;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) mb = fmaxf(mb, m_s[w][g]);
      float wgt[WARPS], zb = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        wgt[w] = mb == -INFINITY ? 0.f : fast_exp2(m_s[w][g] - mb);   // (0 for a warp without keys)
        zb = fmaf(z_s[w][g], wgt[w], zb);
      }
      const bool none = zb == 0.f;                                    // no key at all, or none above -inf (NaN stays NaN)
      const float inv = none ? 0.f : 1.f / zb, lse2 = none ? -INFINITY : mb + log2f(zb);
      const int h = hd * G + g;
      const long long slot = ((long long)(a.slot0 + split) * a.n_rows + row) * a.H + h;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        float a0 = 0.f, a1 = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          const float2 v = w == warp ? make_float2(own[i][2 * rr], own[i][2 * rr + 1]) : part_s(warp, w, i)[rr];
          a0 = fmaf(v.x, wgt[w], a0);
          a1 = fmaf(v.y, wgt[w], a1);
        }
        const int d = (warp * kOwn + i) * 8 + tig * 2;
        if (a.cluster) *reinterpret_cast<float2*>(base_ptr + kResult + (g * D + d) * 4) = make_float2(a0 * inv, a1 * inv);
        else if (a.n_slots == 1) *reinterpret_cast<__nv_bfloat162*>(a.out + (row * a.H + h) * D + d) = __floats2bfloat162_rn(a0 * inv, a1 * inv);
        else *reinterpret_cast<float2*>(a.part_o + slot * D + d) = make_float2(a0 * inv, a1 * inv);
      }
      if (warp == 0 && tig == 0) {
        if (a.cluster) *reinterpret_cast<float*>(base_ptr + kResultLse + g * 4) = aborted || !live ? __uint_as_float(0x7fc00000u) : lse2;
        else if (a.n_slots > 1) a.part_lse[slot] = lse2 * kLn2P;
        else if (a.lse_out) a.lse_out[(long long)h * a.n_rows + row] = lse2 * kLn2P;
      }
    }
  }
  if (!a.cluster) return;
  // ---- the merge, four dims of a head per thread, 32 threads to a unit: the cluster's blocks in their order, and the pieces of the row's context
  // that the kernel before has left, in batches whose loads travel together.  The cluster's blocks take the units in turn; warps that are left
  // share a unit's sources where these are more than a batch.  (All of them in the first block's warps: 30 rows of 8 / 2 heads over 59 pieces each 45 us,
  // so 32; 16 rows of 32 / 8 heads over 16 pieces 29.8 and 26.9.) ----
  cluster_sync();
  constexpr int kWarpsAll = kThreads / 32, kBatch = 10, kOwnBatch = 4;
  struct Merged { float mx, den, acc[4]; };
  Merged* merged_s = reinterpret_cast<Merged*>(base_ptr);             // (the ring, and what was exchanged through it, has been read)
  static_assert(kWarpsAll * 32 * sizeof(Merged) <= kResult, "in front of the results");
  const int pieces = ct.pieces[rc.ctx], quads = G * D / 4, per_block = a.merge_units, across = a.merge_across, groups = a.merge_groups;
  const int group = (a.merge_group_of >> (4 * warp)) & 15;
  const long long stride = a.n_rows * a.H;
  for (int u0 = 0; u0 < per_block; u0 += across) {                    // (once, unless there are more units than warps)
    const int unit_in = u0 + warp - group * across, i = (split * per_block + unit_in) * 32 + lane;
    const bool has = live && fits && !gave_up && group < groups && unit_in < per_block && i < quads;
    const int g = i / (D / 4), d = 4 * (i - g * (D / 4)), h = hd * G + g;
    const long long at = row * a.H + h;
    Merged r = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    auto take = [&](const float* lse, const float4* v, auto count) {
      constexpr int N = decltype(count)::value;
      float m_new = r.mx;
#pragma unroll
      for (int u = 0; u < N; ++u) m_new = fmaxf(m_new, lse[u]);
      const float alpha = r.mx == -INFINITY ? 0.f : fast_exp2(r.mx - m_new);
      r.mx = m_new;
      r.den *= alpha;
#pragma unroll
      for (int e = 0; e < 4; ++e) r.acc[e] *= alpha;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const float w = lse[u] == -INFINITY ? 0.f : fast_exp2(lse[u] - r.mx);    // (NaN stays NaN: logits that were, or a block that gave up)
        r.den += w;
        if (w != 0.f) {
          r.acc[0] = fmaf(w, v[u].x, r.acc[0]); r.acc[1] = fmaf(w, v[u].y, r.acc[1]);
          r.acc[2] = fmaf(w, v[u].z, r.acc[2]); r.acc[3] = fmaf(w, v[u].w, r.acc[3]);
        }
      }
    };
    // (the first batch of pieces is asked for before the cluster's results are read)
    for (int s0 = group; has && (s0 == group || s0 < pieces); s0 += kBatch * groups) {
      float lse[kBatch];
      float4 v[kBatch];
      if (pieces > 0) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int s = s0 + u * groups;
          lse[u] = s < pieces ? a.part_lse[s * stride + at] * kLog2eP : -INFINITY;
          v[u] = s < pieces ? *reinterpret_cast<const float4*>(a.part_o + (s * stride + at) * D + d) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
      if (s0 == group) {
        for (int q0 = group; q0 < a.n_splits; q0 += kOwnBatch * groups) {
          float own_lse[kOwnBatch];
          float4 own_v[kOwnBatch];
#pragma unroll
          for (int u = 0; u < kOwnBatch; ++u) {
            const int s = q0 + u * groups;
            own_lse[u] = -INFINITY;
            own_v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s < a.n_splits) {
              const uint32_t peer = mapa_shared(base, (uint32_t)s);
              own_lse[u] = ld_cluster_f32(peer + kResultLse + g * 4);
              own_v[u] = ld_cluster_f32x4(peer + kResult + (g * D + d) * 4);
            }
          }
          take(own_lse, own_v, std::integral_constant<int, kOwnBatch>{});
        }
      }
      if (pieces > 0) take(lse, v, std::integral_constant<int, kBatch>{});
    }
    if (groups > 1) {                                                 // (then this loop has one trip)
      if (group > 0) merged_s[threadIdx.x] = r;
      __syncthreads();
      if (has && group == 0) {
        for (int x = 1; x < groups; ++x) {
          const Merged& o = merged_s[threadIdx.x + 32 * across * x];
          const float m_new = fmaxf(r.mx, o.mx);
          const float wr = r.mx == -INFINITY ? 0.f : fast_exp2(r.mx - m_new), wo = o.mx == -INFINITY ? 0.f : fast_exp2(o.mx - m_new);
          r.mx = m_new;
          r.den = r.den * wr + o.den * wo;
#pragma unroll
          for (int e = 0; e < 4; ++e) r.acc[e] = r.acc[e] * wr + o.acc[e] * wo;
        }
      }
    }
    if (has && group == 0) {
      const float inv = r.den == 0.f ? 0.f : 1.f / r.den;
      const __nv_bfloat162 lo = __floats2bfloat162_rn(r.acc[0] * inv, r.acc[1] * inv), hi = __floats2bfloat162_rn(r.acc[2] * inv, r.acc[3] * inv);
      *reinterpret_cast<uint2*>(a.out + at * D + d) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      if (d == 0 && a.lse_out) a.lse_out[(long long)h * a.n_rows + row] = r.den == 0.f ? -INFINITY : (r.mx + log2f(r.den)) * kLn2P;
    }
  }
  cluster_sync();                                                     // nobody leaves while its results are read
}

// One warp per (row, head): the slots' weights from their log-sum-exps, then their outputs in slot order.  A launch of few rows is a chain of
// latencies, so the first U outputs, the log-sum-exps and the row's place are asked for side by side.  (Four outputs at a time instead of twenty:
// eight rows of 32 / 8 heads over 6 K and 30 K with 4000 tokens of their own 38.2 / 54.0 us, 36.0 / 54.3 so; one row 20.9 / 36.1, 19.3 / 34.9 so.)
constexpr int kMergeWarps = 4;
template <int D>
__global__ void __launch_bounds__(kMergeWarps * 32)
continuation_merge_kernel(const __grid_constant__ ContTable ct, const __grid_constant__ PagedAttnArgs a, DeviceStatus* st) {
  constexpr int kPer = D / 32, U = 20;
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kMergeWarps + (threadIdx.x >> 5), row = w / a.H;
  const int h = (int)(w - row * a.H);
  griddep_launch();
  griddep_wait();
  if (row >= a.n_rows) return;
  const int status = *reinterpret_cast<volatile int*>(&st->status);
  const long long stride = a.n_rows * a.H, at = row * a.H + h;
  const float* part = a.part_o + at * D + lane * kPer;
  auto load = [&](int s, float* v) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) v[e] = 0.f;
    if (s >= a.n_slots) return;
    if constexpr (kPer == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(part + s * stride * D);
    else *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(part + s * stride * D);
  };
  float v[U][kPer];
#pragma unroll
  for (int u = 0; u < U; ++u) load(u, v[u]);
  // at most 64 slots, two per lane: the pieces of the row's context, then those of its own keys
  float l0 = lane < a.n_slots ? a.part_lse[lane * stride + at] : -INFINITY;
  float l1 = lane + 32 < a.n_slots ? a.part_lse[(lane + 32) * stride + at] : -INFINITY;
  const RowCheck rc = check_row(a, ct, row, h == 0 && lane == 0, st);
  if (rc.seq < 0 || status == RELAXKV_ERR_TIMEOUT) return;
  const int pieces = ct.pieces[rc.ctx];                 // slots between these and the row's own were not written
  if (lane >= pieces && lane < a.slot0) l0 = -INFINITY;
  if (lane + 32 >= pieces && lane + 32 < a.slot0) l1 = -INFINITY;
  const float mx = warp_reduce_max(fmaxf(l0, l1));
  const float w0 = l0 == -INFINITY ? 0.f : __expf(l0 - mx), w1 = l1 == -INFINITY ? 0.f : __expf(l1 - mx);
  const float den = warp_reduce_sum(w0 + w1);
  float acc[kPer];
#pragma unroll
  for (int e = 0; e < kPer; ++e) acc[e] = 0.f;
  for (int s0 = 0; s0 < a.n_slots; s0 += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u;
      const float wgt = __shfl_sync(0xffffffffu, s < 32 ? w0 : w1, s & 31);
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] = wgt != 0.f ? fmaf(wgt, v[u][e], acc[e]) : acc[e];      // (an empty piece's output is not looked at)
    }
    if (s0 + U < a.n_slots) {
#pragma unroll
      for (int u = 0; u < U; ++u) load(s0 + U + u, v[u]);
    }
  }
  const float inv = den != 0.f ? 1.f / den : 0.f;
  uint32_t packed[kPer / 2];
#pragma unroll
  for (int e = 0; e < kPer; e += 2) {
    const __nv_bfloat162 v2 = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
    packed[e / 2] = *reinterpret_cast<const uint32_t*>(&v2);
  }
  uint16_t* o = a.out + at * D + lane * kPer;
  if constexpr (kPer == 4) *reinterpret_cast<uint2*>(o) = make_uint2(packed[0], packed[1]);
  else *reinterpret_cast<uint32_t*>(o) = packed[0];
  if (lane == 0 && a.lse_out) a.lse_out[(long long)h * a.n_rows + row] = den != 0.f ? mx + logf(den) : -INFINITY;
}

template <int D, int GMAX, int WARPS>
static relaxkv_status launch_paged_g(const CUtensorMap* maps, const ContTable& ct, PagedAttnArgs a, DeviceStatus* st, cudaStream_t stream) {
  static std::atomic<int> attr_done[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return RELAXKV_ERR_CUDA;
  using L = PagSmem<D, WARPS>;
  auto kern = paged_attention_kernel<D, GMAX, WARPS>;
  if (!attr_done[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynamic) != cudaSuccess) return RELAXKV_ERR_CUDA;
    attr_done[dev].store(1, std::memory_order_release);
  }
  const long long blocks = a.n_rows * a.n_splits * a.Hkv;
  if (blocks > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (a.cluster) {                                       // who merges what: the kernel's divisions
    constexpr int kWarpsAll = L::kThreads / 32;
    int most = 0;
    for (int b = 0; b < ct.n_req; ++b) most = std::max(most, ct.pieces[b]);
    a.merge_units = ((a.H / a.Hkv * D / 4 + 31) / 32 + a.n_splits - 1) / a.n_splits;
    a.merge_across = std::min(a.merge_units, kWarpsAll);
    a.merge_groups = std::max(1, std::min(kWarpsAll / a.merge_units, (a.n_splits + most + 9) / 10));
    for (int w = 0; w < kWarpsAll; ++w) a.merge_group_of |= (uint32_t)(w / a.merge_across) << (4 * w);
  }
  const int pieces = a.cluster ? a.n_splits : 1;
  return cuda_ok(launch_chained_clusters(pieces, kern, dim3((unsigned)blocks), L::kThreads, L::kDynamic, stream, maps[0], maps[1], maps[2], maps[3], ct, a, st));
}

template <int D>
static relaxkv_status launch_paged_d(int warps, const CUtensorMap* maps, const ContTable& ct, const PagedAttnArgs& a, DeviceStatus* st, cudaStream_t stream) {
  if (a.H / a.Hkv > 8)
    return warps == 1 ? launch_paged_g<D, 16, 1>(maps, ct, a, st, stream)
                      : warps == 2 ? launch_paged_g<D, 16, 2>(maps, ct, a, st, stream) : launch_paged_g<D, 16, 4>(maps, ct, a, st, stream);
  return warps == 1 ? launch_paged_g<D, 8, 1>(maps, ct, a, st, stream)
                    : warps == 2 ? launch_paged_g<D, 8, 2>(maps, ct, a, st, stream) : launch_paged_g<D, 8, 4>(maps, ct, a, st, stream);
}

template <int D, int GMAX>
static int clusters_at_once(int n, int sms) {
  static std::atomic<int> known[kMaxDevices][kPagCluster + 1];
  int dev = 0;
  const int guess = std::max(1, 2 * sms / n - sms / 16);
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return guess;
  int k = known[dev][n].load(std::memory_order_acquire);
  if (k > 0) return k;
  using L = PagSmem<D, 4>;
  auto kern = paged_attention_kernel<D, GMAX, 4>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(n * sms));
  cfg.blockDim = L::kThreads;
  cfg.dynamicSmemBytes = L::kDynamic;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)n; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynamic) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&k, kern, &cfg) != cudaSuccess || k < 1) {
    (void)cudaGetLastError();
    k = guess;
  }
  known[dev][n].store(k, std::memory_order_release);
  return k;
}

int cluster_that_fits(const relaxkv_shape* shape, int n, long long items) {
  const int sms = std::max(1, sm_count_of_current_device());
  const bool wide = shape->n_q_heads / shape->n_kv_heads > 8;
  for (; n > 1; --n) {
    const int room = shape->head_dim == 128 ? (wide ? clusters_at_once<128, 16>(n, sms) : clusters_at_once<128, 8>(n, sms))
                                            : (wide ? clusters_at_once<64, 16>(n, sms) : clusters_at_once<64, 8>(n, sms));
    if (items <= room) break;
  }
  return n;
}

relaxkv_status launch_paged_attention(const relaxkv_shape* shape, const relaxkv_cache_view* cache, const relaxkv_paged_cache* store,
                                      const ContTable& ct, PagedAttnArgs a, cudaStream_t stream) {
  DeviceStatus* st = status_word();
  if (!st) return RELAXKV_ERR_CUDA;
  const int D = shape->head_dim;
  const int sms = sm_count_of_current_device();
  if (sms <= 0) return RELAXKV_ERR_CUDA;
  const int warps = a.n_splits == 1 ? paged_warps(a.n_rows * a.Hkv, (long long)a.listed_most * a.ctx_block + a.max_len, sms) : 4;
  CUtensorMap maps[4] = {};
  if (a.ctx_keys != CTX_KEYS_NONE) {
    long long tokens = 0;
    for (int b = 0; b < ct.n_req; ++b) tokens = std::max(tokens, ct.ctx_len[b] ? ct.tok_off[b] + ct.ctx_len[b] : 0);
    const uint32_t box = (uint32_t)std::min(a.ctx_block, 16 * warps);
    for (int i = 0; i < 2; ++i)
      if (!make_block_map(&maps[i], i ? cache->v : cache->k, D, (uint64_t)tokens, a.Hkv, 1, (uint64_t)cache->token_stride, (uint64_t)cache->head_stride,
                          (uint64_t)cache->token_stride, box)) return RELAXKV_ERR_CUDA;
  }
  if (a.max_len > 0) {
    const uint32_t box = (uint32_t)std::min(a.page, 16 * warps);
    for (int i = 0; i < 2; ++i)
      if (!make_block_map(&maps[2 + i], i ? store->v : store->k, D, (uint64_t)store->block_size, a.Hkv, (uint64_t)store->n_blocks,
                          (uint64_t)store->token_stride, (uint64_t)store->head_stride, (uint64_t)store->block_stride, box)) return RELAXKV_ERR_CUDA;
  }
  return D == 128 ? launch_paged_d<128>(warps, maps, ct, a, st, stream) : launch_paged_d<64>(warps, maps, ct, a, st, stream);
}

relaxkv_status launch_continuation_merge(const ContTable& ct, const PagedAttnArgs& a, int D, cudaStream_t stream) {
  DeviceStatus* st = status_word();
  if (!st) return RELAXKV_ERR_CUDA;
  const long long warps = a.n_rows * a.H;
  auto kern = D == 128 ? continuation_merge_kernel<128> : continuation_merge_kernel<64>;
  return cuda_ok(launch_chained(kern, dim3((unsigned)((warps + kMergeWarps - 1) / kMergeWarps)), kMergeWarps * 32, 0, stream, ct, a, st));
}

}  // namespace relaxkv
