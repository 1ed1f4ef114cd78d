// Attention of a step's rows over the context they share, read once for all of them (relaxkv_shared_prefix_attention).
//
// Rows x heads of a group meet the same keys, so they are the rows of a matrix product: a block owns 128 of them (128 / G rows of the step),
// one KV head and a piece of the context, and walks it in 128-key tiles: TMA (128-byte swizzle) -> S = Q K^T (tcgen05, accumulators in tensor
// memory) -> softmax warps (thread = row), P as bf16 over S -> O += P V (tcgen05, P from tensor memory).  S of the next tile is issued before
// O of this one, so the tensor pipe works while the softmax does.  With up to 128 rows the kernel is bound by the bytes of K and V (a tile
// of 64 KB takes an SM's share of HBM 1.5 us, its products and exponentials half of that), with more by the exponentials.  The pieces' results are
// merged with those of the rows' own tokens by their log-sum-exps.  Every wait is bounded.
#include "continuation_splits.cuh"
#include "paged_attention.cuh"
#include "sm100_ptx.cuh"
#include <atomic>

namespace relaxkv {

using namespace ptx;

constexpr int kPreTile = 128;                         // keys per tile = rows per block
constexpr int kPreRing = 6;                           // tile buffers, used in the order K0 V0 K1 V1 ...
constexpr int kPreThreads = 192;                      // four softmax warps, the TMA warp, the MMA warp
constexpr float kPreRescale = 8.0f;                   // log2 units: O is rescaled only when the row maximum grew by more
constexpr float kLog2ePre = 1.4426950408889634f, kLn2Pre = 0.6931471805599453f;

template <int D>
struct PreSmem {
  static constexpr int kHalves = D / 64;
  static constexpr int kHalfBytes = kPreTile * 128;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kQ = 0;
  static constexpr int kKV = kTileBytes;
  static constexpr int kBar = kKV + kPreRing * kTileBytes;
  static constexpr int kNumBars = 2 * kPreRing + 9;   // full, empty | q, s[2], p_lo[2], p_hi[2], o, vfix
  static constexpr int kMisc = kBar + 8 * kNumBars;   // tensor memory address, abort flag
  static constexpr int kTotal = kMisc + 16;
  static constexpr int kDynamic = kTotal + 1024;
};

// P of keys [32 C0, 32 C1): p = 2^(s * scale - m) as bf16 over S, and its sum.
template <int C0, int C1>
__device__ __forceinline__ float prefix_exponentials(uint32_t t_s, const uint32_t* s, float scale, float neg_m) {
  float z0 = 0.f, z1 = 0.f, z2 = 0.f, z3 = 0.f;
#pragma unroll
  for (int c = C0; c < C1; ++c) {
    uint32_t pk[16];
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      float x[4], p[4];
#pragma unroll
      for (int e = 0; e < 4; e += 2)
        fma2(x[e], x[e + 1], __uint_as_float(s[c * 32 + i + e]), __uint_as_float(s[c * 32 + i + e + 1]), scale, scale, neg_m, neg_m);
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = fast_exp2(x[e]);
      add2(z0, z1, p[0], p[1]);
      add2(z2, z3, p[2], p[3]);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(p[e], p[e + 1]);
        pk[(i + e) >> 1] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    tmem_st16(t_s + c * 16, pk);
  }
  return (z0 + z1) + (z2 + z3);
}

template <int D>
__global__ void __launch_bounds__(kPreThreads, 1)
prefix_attention_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ContTable ct,
                        const __grid_constant__ PagedAttnArgs a, int rows_per_tile, DeviceStatus* st) {
  using L = PreSmem<D>;
  constexpr uint32_t kTmemCols = 512;                   // S of even tiles | S of odd tiles | O
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar_full = base + L::kBar, bar_empty = bar_full + 8 * kPreRing, bar_q = bar_empty + 8 * kPreRing, bar_s = bar_q + 8,
                 bar_plo = bar_s + 16, bar_phi = bar_plo + 16, bar_o = bar_phi + 16, bar_vfix = bar_o + 8;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + L::kMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + L::kMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.H / a.Hkv;
  // which context, rows, head and piece: the row tiles of a piece stand side by side and find its keys in L2
  const int b = find_segment(ct.tile_cu, ct.n_req, (int)blockIdx.x);
  const int n_rt = (ct.max_rows[b] + rows_per_tile - 1) / rows_per_tile, at = (int)blockIdx.x - ct.tile_cu[b];
  const int rt = at % n_rt, hd = at / n_rt % a.Hkv, piece = at / (n_rt * a.Hkv);
  const int ctx_len = ct.ctx_len[b], n_tiles = (ctx_len + kPreTile - 1) / kPreTile;
  const int per = (n_tiles + ct.pieces[b] - 1) / ct.pieces[b], j0 = min(n_tiles, piece * per), n = min(n_tiles, j0 + per) - j0;
  if (threadIdx.x == 128) { prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v); }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kPreRing; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
    mbar_init(bar_q, 128);
    mbar_init(bar_s, 1); mbar_init(bar_s + 8, 1);
    for (int x = 0; x < 2; ++x) { mbar_init(bar_plo + 8 * x, 128); mbar_init(bar_phi + 8 * x, 128); }
    mbar_init(bar_o, 1);
    mbar_init(bar_vfix, 32);
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  griddep_wait();
  const int status = *reinterpret_cast<volatile int*>(&st->status);
  const long long row0 = a.row_cu[ct.seq_cu[b]], row1 = a.row_cu[ct.seq_cu[b + 1]];
  const long long first = row0 + (long long)rt * rows_per_tile;
  if (row0 < 0 || row1 > a.n_rows || row1 - row0 > ct.max_rows[b]) {        // more rows than the host's bounds: report, touch nothing
    if (threadIdx.x == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_PREFIX_ATTN, (int)(row1 - row0), b);
    return;
  }
  if (first >= row1 || status == RELAXKV_ERR_TIMEOUT) return;
  const int n_rows = (int)min((long long)rows_per_tile, row1 - first);
  if (warp == 5) { tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch();                                     // (the block holds its tensor memory)
  const uint32_t tmem_base = *tmem_slot;
  const int tail = ctx_len % kPreTile;                  // tokens of the context's last tile, 0: all
  const bool fix_v = tail != 0 && j0 + n == n_tiles && n > 0;

  if (warp == 4) {
    // ================= TMA producer =================
    if (lane == 0) {
      const int token0 = (int)ct.tok_off[b] + j0 * kPreTile;
      for (int u = 0; u < 2 * n; ++u) {
        const int s = u % kPreRing;
        if (u >= kPreRing && !mbar_wait(bar_empty + 8 * s, (uint32_t)(u / kPreRing - 1) & 1, abort_flag)) break;
        mbar_expect_tx(bar_full + 8 * s, L::kTileBytes);
        tma_load_5d(base + L::kKV + s * L::kTileBytes, (u & 1) ? &tm_v : &tm_k, bar_full + 8 * s, token0 + (u >> 1) * kPreTile, hd, 0);
      }
    }
    __syncwarp();
    if (fix_v) {
      // V rows behind the context belong to nobody (0 x NaN = NaN on the tensor core): zero them once their tile has landed
      const int u = 2 * n - 1, s = u % kPreRing;
      if (mbar_wait(bar_full + 8 * s, (uint32_t)(u / kPreRing) & 1, abort_flag)) {
        uint8_t* vt = base_ptr + L::kKV + s * L::kTileBytes;
        for (int i = lane; i < (kPreTile - tail) * 8 * L::kHalves; i += 32) {
          const int c = i & 7, r = tail + (i >> 3) % (kPreTile - tail), hf = (i >> 3) / (kPreTile - tail);
          *reinterpret_cast<uint4*>(vt + hf * L::kHalfBytes + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      mbar_arrive(bar_vfix);
    }
  } else if (warp == 5) {
    // ================= MMA issuer =================
    if (lane == 0 && n > 0) {
      constexpr uint32_t idesc_qk = idesc_bf16_f32(kPreTile, kPreTile, 0), idesc_pv = idesc_bf16_f32(kPreTile, D, 1);
      const uint32_t hi = desc_hi_sw128(1024);
      auto issue_qk = [&](int j) -> bool {              // S_j = Q K_j^T
        const int u = 2 * j, s = u % kPreRing;
        if (!mbar_wait(bar_full + 8 * s, (uint32_t)(u / kPreRing) & 1, abort_flag)) return false;
        tc_fence_after();
#pragma unroll
        for (int hf = 0; hf < L::kHalves; ++hf)
          mma_ss_4steps(tmem_base + (j & 1) * 128, desc_lo(base + L::kQ + hf * L::kHalfBytes, 16),
                        desc_lo(base + L::kKV + s * L::kTileBytes + hf * L::kHalfBytes, 16), hi, idesc_qk, hf > 0 ? 1u : 0u);
        mma_commit(bar_s + 8 * (j & 1));
        mma_commit(bar_empty + 8 * s);
        return true;
      };
      bool ok = mbar_wait(bar_q, 0, abort_flag) && issue_qk(0);
      for (int j = 0; ok && j < n; ++j) {
        if (j + 1 < n && !(ok = issue_qk(j + 1))) break;
        const int u = 2 * j + 1, s = u % kPreRing;
        if (!(ok = mbar_wait(bar_full + 8 * s, (uint32_t)(u / kPreRing) & 1, abort_flag))) break;
        if (fix_v && j == n - 1 && !(ok = mbar_wait(bar_vfix, 0, abort_flag))) break;
        if (!(ok = mbar_wait(bar_plo + 8 * (j & 1), (uint32_t)(j >> 1) & 1, abort_flag))) break;
        tc_fence_after();
        const uint32_t v_lo = desc_lo(base + L::kKV + s * L::kTileBytes, L::kHalfBytes), p = tmem_base + (j & 1) * 128;
        mma_ts_steps<6>(tmem_base + 256, p, v_lo, hi, idesc_pv, j > 0 ? 1u : 0u);       // the first 96 keys while the last 32 are worked on
        if (!(ok = mbar_wait(bar_phi + 8 * (j & 1), (uint32_t)(j >> 1) & 1, abort_flag))) break;
        tc_fence_after();
        mma_ts_steps<2>(tmem_base + 256, p + 48, v_lo + 6 * 128, hi, idesc_pv, 1u);
        mma_commit(bar_empty + 8 * s);
        mma_commit(bar_o);
      }
    }
  } else {
    // ================= softmax: thread = (row of the step, head) = TMEM lane =================
    const int t_local = (int)threadIdx.x / G, head = hd * G + (int)threadIdx.x - t_local * G;
    const bool mine = t_local < n_rows;
    const long long row = first + t_local;
    {
      uint8_t* q_s = base_ptr + L::kQ + threadIdx.x * 128;
      const uint4* q = reinterpret_cast<const uint4*>(a.q + (row * a.H + head) * D);
#pragma unroll
      for (int c = 0; c < D / 8; ++c)
        *reinterpret_cast<uint4*>(q_s + (c >> 3) * L::kHalfBytes + (((c & 7) ^ ((int)threadIdx.x & 7)) << 4)) = mine ? q[c] : make_uint4(0, 0, 0, 0);
      fence_proxy_async_smem();
      mbar_arrive(bar_q);
    }
    const bool busy = __any_sync(0xffffffffu, mine);    // a warp without rows only keeps step
    const uint32_t lane_base = tmem_base + ((uint32_t)(warp * 32) << 16), t_o = lane_base + 256;
    float m = -1.0e30f, z = 0.f;                        // (finite, so that logits of -inf leave 2^(-inf) = 0)
    bool ok = true;
    for (int j = 0; j < n; ++j) {
      ok = mbar_wait(bar_s + 8 * (j & 1), (uint32_t)(j >> 1) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      if (busy) {
        const uint32_t t_s = lane_base + (j & 1) * 128;
        uint32_t s[kPreTile];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, &s[c * 32]);
        tmem_wait_ld();
        const int limit = ctx_len - (j0 + j) * kPreTile;
        if (limit < kPreTile) {
#pragma unroll
          for (int i = 0; i < kPreTile; ++i)
            if (i >= limit) s[i] = 0xff800000u;         // -inf
        }
        float mx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = fmaxf(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
#pragma unroll
        for (int i = 16; i < kPreTile; i += 2) mx[(i >> 1) & 7] = fmax3(mx[(i >> 1) & 7], __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
        const float m_new = fmax3(fmax3(mx[0], mx[1], mx[2]), fmax3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * a.scale_log2;
        const float m_old = m;
        const bool need = m_new > m + kPreRescale;
        if (need) m = m_new;
        if (j > 0 && __any_sync(0xffffffffu, need)) {
          ok = mbar_wait(bar_o, (uint32_t)(j - 1) & 1, abort_flag);           // O of the tile before is complete
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          const float alpha = fast_exp2(m_old - m);
          z *= alpha;
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32(t_o + c * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
            tmem_st32(t_o + c * 32, o);
          }
        }
        z += prefix_exponentials<0, 3>(t_s, s, a.scale_log2, -m);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(bar_plo + 8 * (j & 1));
        z += prefix_exponentials<3, 4>(t_s, s, a.scale_log2, -m);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(bar_phi + 8 * (j & 1));
      } else {
        tc_fence_before();
        mbar_arrive(bar_plo + 8 * (j & 1));
        mbar_arrive(bar_phi + 8 * (j & 1));
      }
    }
    if (ok && n > 0) {
      ok = mbar_wait(bar_o, (uint32_t)(n - 1) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
    }
    if (ok && busy) {
      const bool none = z == 0.f;                       // no key, or none of a logit above -inf (NaN stays NaN)
      const float inv = none ? 0.f : 1.f / z, lse = none ? -INFINITY : (m + log2f(z)) * kLn2Pre;
      const bool direct = a.n_slots == 1;
      const bool store = mine && (!direct || check_row(a, ct, row, true, st).seq >= 0);
      const long long slot = ((long long)piece * a.n_rows + row) * a.H + head;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        if (n > 0) { tmem_ld32(t_o + c * 32, o); tmem_wait_ld(); }
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = none ? 0u : __float_as_uint(__uint_as_float(o[i]) * inv);
        if (store && direct) {
          uint16_t* p = a.out + (row * a.H + head) * D + c * 32;
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const __nv_bfloat162 h2 = __floats2bfloat162_rn(__uint_as_float(o[i + 2 * e]), __uint_as_float(o[i + 2 * e + 1]));
              w[e] = *reinterpret_cast<const uint32_t*>(&h2);
            }
            *reinterpret_cast<uint4*>(p + i) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else if (store) {
          float* p = a.part_o + slot * D + c * 32;
#pragma unroll
          for (int i = 0; i < 32; i += 8) st_global_32b(p + i, o + i);        // (the workspace is 256-byte aligned)
        }
      }
      if (store && direct && a.lse_out) a.lse_out[(long long)head * a.n_rows + row] = lse;
      if (store && !direct) a.part_lse[slot] = lse;
    }
  }
  // ---- teardown ----
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0) report(st, RELAXKV_ERR_TIMEOUT, KID_PREFIX_ATTN, (int)blockIdx.x, hd);
    const uint64_t t0 = global_timer_ns();              // copies and products still in flight: let them land
    while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 5) { tc_fence_after(); tmem_dealloc(tmem_base, kTmemCols); }
}

template <int D>
static relaxkv_status launch_prefix(const relaxkv_cache_view* cache, const ContTable& ct, const PagedAttnArgs& a, int rows_per_tile, cudaStream_t stream) {
  DeviceStatus* st = status_word();
  if (!st) return RELAXKV_ERR_CUDA;
  static std::atomic<int> attr_done[kMaxDevices];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return RELAXKV_ERR_CUDA;
  if (!attr_done[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(prefix_attention_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, PreSmem<D>::kDynamic) != cudaSuccess)
      return RELAXKV_ERR_CUDA;
    attr_done[dev].store(1, std::memory_order_release);
  }
  long long tokens = 0;
  for (int b = 0; b < ct.n_req; ++b) tokens = std::max(tokens, ct.ctx_len[b] ? ct.tok_off[b] + ct.ctx_len[b] : 0);
  CUtensorMap tm[2];
  for (int i = 0; i < 2; ++i)
    if (!make_block_map(&tm[i], i ? cache->v : cache->k, D, (uint64_t)tokens, a.Hkv, 1, (uint64_t)cache->token_stride, (uint64_t)cache->head_stride,
                        (uint64_t)cache->token_stride, kPreTile)) return RELAXKV_ERR_CUDA;
  return cuda_ok(launch_chained(prefix_attention_kernel<D>, dim3((unsigned)ct.tile_cu[ct.n_req]), kPreThreads, PreSmem<D>::kDynamic, stream, tm[0], tm[1],
                                ct, a, rows_per_tile, st));
}

// Checks that the attention calls share.  Fills ct and what of `a` does not depend on how the keys are cut.
static relaxkv_status prepare_continuations(const relaxkv_shape* shape, const relaxkv_cache_view* cache, const relaxkv_paged_cache* store,
                                            const relaxkv_continuation_rows* rows, int ctx_block, const void* q, void* out, float* lse_out,
                                            void* workspace, size_t workspace_bytes, ContTable& ct, PagedAttnArgs& a) {
  relaxkv_status rc = check_contexts(shape);
  if (rc != RELAXKV_OK) return rc;
  bool any_ctx = false;
  for (int b = 0; b < shape->n_req; ++b) any_ctx |= shape->h_ctx_len[b] > 0;
  if (any_ctx && (rc = check_cache(shape, cache, true)) != RELAXKV_OK) return rc;
  fill_contexts(ct, shape, any_ctx ? cache : nullptr, ctx_block);
  if ((rc = check_rows(shape, rows, true, ct)) != RELAXKV_OK) return rc;
  if (rows->max_len > 0 && (rc = check_store(store, shape->head_dim)) != RELAXKV_OK) return rc;
  if (!q || !out || !workspace || !aligned16(q) || !aligned16(out)) return RELAXKV_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return RELAXKV_ERR_INVALID_ARG;
  const ContWs ws = cont_ws(shape, rows->n_rows, 0);
  if (workspace_bytes < ws.total) return RELAXKV_ERR_WORKSPACE_TOO_SMALL;
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.lse_out = lse_out;
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.part_o);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + ws.part_lse);
  a.row_seq = rows->row_seq; a.row_len = rows->row_len; a.row_cu = rows->row_cu; a.table = rows->block_table;
  a.table_stride = rows->table_stride; a.n_rows = rows->n_rows; a.table_width = rows->table_width; a.max_len = rows->max_len;
  a.n_blocks = rows->max_len > 0 ? store->n_blocks : 0;
  a.page = rows->max_len > 0 ? store->block_size : kPreTile;
  a.ctx_block = kPreTile;
  a.H = shape->n_q_heads; a.Hkv = shape->n_kv_heads; a.n_seq = rows->n_seq;
  a.scale_log2 = shape->softmax_scale * kLog2ePre;
  return RELAXKV_OK;
}

}  // namespace relaxkv

using namespace relaxkv;

extern "C" size_t relaxkv_continuation_workspace_bytes(const relaxkv_shape* shape, int64_t n_rows, int32_t block_size) {
  if (check_contexts(shape) != RELAXKV_OK || n_rows < 0 || n_rows > 0x7fffffffLL / (shape->n_q_heads * 2)) return 0;
  if (block_size != 0 && !block_size_ok(block_size)) return 0;
  return cont_ws(shape, n_rows, block_size).total;
}

extern "C" relaxkv_status relaxkv_shared_prefix_attention(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, const relaxkv_paged_cache* store, const relaxkv_continuation_rows* rows,
    const void* q, void* out, float* lse_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_shared_prefix_attention");
  ContTable ct;
  PagedAttnArgs a = {};
  relaxkv_status rc = prepare_continuations(shape, cache, store, rows, 0, q, out, lse_out, workspace, workspace_bytes, ct, a);
  if (rc != RELAXKV_OK || rows->n_rows == 0) return rc;
  const int sms = sm_count_of_current_device();
  if (sms <= 0) return RELAXKV_ERR_CUDA;
  const int D = shape->head_dim, rows_per_tile = kPreTile / (a.H / a.Hkv), slots = cont_slots(a.n_rows);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // ---- pieces of the rows' own keys (0: there are none), and of the contexts ----
  const bool own = a.max_len > 0;
  const int own_pieces = own ? paged_pieces(a.n_rows * a.Hkv, (a.max_len + 63) / 64, sms, std::max(1, slots / 4)) : 0;
  int n_tiles[kMaxReqInline], row_tiles[kMaxReqInline], most = 0;
  for (int b = 0; b < ct.n_req; ++b) {
    n_tiles[b] = (int)(((long long)ct.ctx_len[b] + kPreTile - 1) / kPreTile);
    row_tiles[b] = ct.ctx_len[b] > 0 ? (ct.max_rows[b] + rows_per_tile - 1) / rows_per_tile : 0;
  }
  // a slot more is written and read once: 8 bytes per element at some 5 TB/s, against 1.5 us for a tile
  const double merge_tiles = (double)a.n_rows * a.H * D * 8 / 5.0e12 / 1.5e-6;
  const int per = prefix_tiles_per_block(n_tiles, row_tiles, ct.n_req, a.Hkv, sms, slots - own_pieces, merge_tiles);
  long long blocks = 0;
  bool all = true;                                      // every row has a piece
  for (int b = 0; b < ct.n_req; ++b) {
    ct.pieces[b] = row_tiles[b] > 0 ? (n_tiles[b] + per - 1) / per : 0;
    blocks += (long long)row_tiles[b] * a.Hkv * ct.pieces[b];
    if (blocks > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
    ct.tile_cu[b + 1] = (int)blocks;
    most = std::max(most, ct.pieces[b]);
    all &= own || ct.pieces[b] > 0 || ct.max_rows[b] == 0;
  }
  a.slot0 = own ? most : kContSlotsMost;                // without own keys no slot is theirs
  a.n_slots = most + own_pieces;
  a.n_splits = own_pieces;
  if (a.n_slots <= 1 && !all) a.n_slots = 2;            // rows without any key: the merge writes their zeros
  if (most > 0) {
    rc = D == 128 ? launch_prefix<128>(cache, ct, a, rows_per_tile, s) : launch_prefix<64>(cache, ct, a, rows_per_tile, s);
    if (rc != RELAXKV_OK) return rc;
  }
  if (own && (rc = launch_paged_attention(shape, cache, store, ct, a, s)) != RELAXKV_OK) return rc;
  return a.n_slots == 1 ? RELAXKV_OK : launch_continuation_merge(ct, a, D, s);
}

extern "C" relaxkv_status relaxkv_block_sparse_attention(
    const relaxkv_shape* shape, const relaxkv_cache_view* cache, const relaxkv_paged_cache* store, const relaxkv_continuation_rows* rows,
    int32_t block_size, const int32_t* blocks, int32_t n_select, const void* q, void* out, float* lse_out, void* workspace, size_t workspace_bytes,
    relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_block_sparse_attention");
  ContTable ct;
  PagedAttnArgs a = {};
  if (!block_size_ok(block_size)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (!blocks || n_select < 1) return RELAXKV_ERR_INVALID_ARG;
  relaxkv_status rc = prepare_continuations(shape, cache, store, rows, block_size, q, out, lse_out, workspace, workspace_bytes, ct, a);
  if (rc != RELAXKV_OK) return rc;
  if (n_select > 0x7fffffff / block_size) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (rows->n_rows == 0) return RELAXKV_OK;
  const int sms = sm_count_of_current_device();
  if (sms <= 0) return RELAXKV_ERR_CUDA;
  bool any_ctx = false;
  for (int b = 0; b < ct.n_req; ++b) any_ctx |= ct.ctx_len[b] > 0;
  a.ctx_keys = any_ctx ? CTX_KEYS_LISTED : CTX_KEYS_NONE;
  a.lists = blocks; a.n_select = n_select; a.ctx_block = block_size;
  const long long tiles = ((long long)n_select * block_size + 63) / 64 + (a.max_len + 63) / 64;
  a.n_splits = paged_pieces(a.n_rows * a.Hkv, tiles, sms, cont_slots(a.n_rows));
  a.slot0 = 0;
  a.n_slots = a.n_splits;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = launch_paged_attention(shape, cache, store, ct, a, s)) != RELAXKV_OK) return rc;
  return a.n_slots == 1 ? RELAXKV_OK : launch_continuation_merge(ct, a, shape->head_dim, s);
}
