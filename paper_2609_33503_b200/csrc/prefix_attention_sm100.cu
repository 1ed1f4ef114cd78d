// Attention of a step's rows over the context they share, read once for all of them (relaxkv_shared_prefix_attention).
//
// Rows x heads of a group meet the same keys, so they are the rows of a matrix product: a block owns 128 of them (128 / G rows of the
// step), one KV head and a piece of the context, and walks it in 128-key tiles: TMA (128-byte swizzle) -> S = Q K^T (tcgen05, Q and the
// accumulators in tensor memory) -> softmax (thread = row) -> P as bf16 in tensor memory -> O += P V (tcgen05).
// With up to 128 rows the kernel is bound by the bytes of K and V: a tile of 64 KB takes an SM's share of HBM 1.5 us.  With several row tiles to
// a context a tile's products (2 x 512 clk), its 16 K exponentials (16 per clk) and its way through shared memory (written once and read
// once at 128 bytes per clk, as long as Q is not read from there, too) all take 1024 clk, so they have to overlap:
//   two groups of four softmax warps take the even and the odd tiles;
//   S is double-buffered and free again as soon as a group has it in registers, so S of tile j + 2 is made while P of tile j is;
//   P and O are single: a group hands its P over when O of the tile before is complete, which is also when O may be rescaled (every barrier
//   belongs to the even or to the odd tiles, so that nobody who waits for one phase can be two behind);
//   the running maximum of a row goes from group to group through shared memory (known a third into a group's step); sums stay with the groups.
// Tiles are loaded in the order of the products, K two tiles ahead of V: with K0 V0 K1 V1 ... a V tile waits in its buffer for two tiles' time, and five
// buffers were too few (64 rows of 40 / 8 heads over 32 K without own tokens 80 us, seven 59; in this order five 55.5, six 57, seven 58).
// Measured: some 1700 clk per tile.  (Each group with an output of its own, S and P in one place, Q in shared memory: 1780.)  64 rows of 40 / 8 heads over
// 32 K, three row tiles: 47 us of the 21 that the keys take and the 30 of the products.  16 rows of 32 / 8 heads over 16 K, where a block has eight
// tiles and its start and end count: 14 us of 10.
// A row's pieces are merged with its own tokens by their log-sum-exps: by the clusters of the kernel over those (paged_attention.cu), or by a kernel
// behind it.  That kernel begins when every block here has passed its wait, and reads what this one writes only after its own: 83.8 -> 80.6 and
// 31.0 -> 29.5 us for whole calls of those two sizes.  Every wait is bounded.
#include "continuation_splits.cuh"
#include "paged_attention.cuh"
#include "sm100_ptx.cuh"
#include <atomic>

namespace relaxkv {

using namespace ptx;

constexpr int kPreTile = 128;                         // keys per tile = rows per block
constexpr int kPreRing = 5;                           // tile buffers, used in the order of the products: K0 K1 K2 V0 K3 V1 ...
constexpr int kPreThreads = 384;                      // two groups of four softmax warps; the TMA warp, the MMA warp, two idle
constexpr float kPreRescale = 8.0f;                   // log2 units: O is rescaled only when the row maximum grew by more
// What a row's maximum begins with: the lowest finite number, so that logits of -inf leave 2^(-inf) = 0 and any finite logit more.
constexpr float kPreLowest = -3.402823466e38f;
// s * scale - m in one rounding keeps what the rounding of m has cut off: the same factor, up to 2^(|m| 2^-24), on all weights of a row, which their
// sum takes out again.  Where the largest logit of a tile is beyond this (2^-9 of a weight), its logits are rounded first, as m is: the factor would
// take a lone weight off 1 as a bf16, and leave the range of numbers where |m| is 2^31.  (A tile below it beside such an m has weights of zero, or
// makes the next m itself.)  Looked at before the other group's maximum is waited for: 64 rows over 32 K 80.7 us, behind it 81.0, without 79.8; 16 over
// 16 K 26.4, 26.7 and 26.4.
constexpr float kPreExact = 32768.f;
constexpr float kLog2ePre = 1.4426950408889634f, kLn2Pre = 0.6931471805599453f;

// p = 2^(s * scale - m) of a row's 128 keys as bf16 pairs, and their sum.  bf16 is what the product with V takes beside bf16 values: its rounding
// errors (up to 2^-8 of a weight, of either sign) average out over the keys; the sum is that of the unrounded weights, in fp32.
__device__ __forceinline__ float prefix_exponentials(const uint32_t* s, uint32_t* pk, float scale, float neg_m) {
  float z0 = 0.f, z1 = 0.f, z2 = 0.f, z3 = 0.f;
#pragma unroll
  for (int i = 0; i < kPreTile; i += 4) {
    float y[4], p[4];
#pragma unroll
    for (int e = 0; e < 4; e += 2)
      fma2(y[e], y[e + 1], __uint_as_float(s[i + e]), __uint_as_float(s[i + e + 1]), scale, scale, neg_m, neg_m);
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = fast_exp2(y[e]);
    add2(z0, z1, p[0], p[1]);
    add2(z2, z3, p[2], p[3]);
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(p[e], p[e + 1]);
      pk[(i + e) >> 1] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return (z0 + z1) + (z2 + z3);
}

// The u-th of a block's 2 n loads: Q K^T is two tiles ahead of P V.
struct PreLoad { int tile; bool v; };
__device__ __forceinline__ PreLoad prefix_load(int u, int n) {
  if (u < min(n, 2)) return {u, false};
  if (u >= 2 * n - 2) return {u - n, true};
  return u & 1 ? PreLoad{(u - 3) >> 1, true} : PreLoad{(u + 2) >> 1, false};
}

template <int D>
struct PreSmem {
  static constexpr int kHalves = D / 64;
  static constexpr int kHalfBytes = kPreTile * 128;
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kBar = kPreRing * kTileBytes;
  static constexpr int kNumBars = 2 * kPreRing + 12;  // full, empty | q, s[2], read[2], p[2], m[2], o[2], vfix
  static constexpr int kMisc = kBar + 8 * kNumBars;   // tensor memory address, abort flag
  static constexpr int kMax = kMisc + 8;              // running maximum of every row
  static constexpr int kSum = kMax + 4 * kPreTile;    // sums of every row, by group
  static constexpr int kTotal = kSum + 8 * kPreTile;
  static constexpr int kDynamic = kTotal + 1024;
  static constexpr int kOutStride = D * 2 + 16;       // bytes between the half rows of partial output that threads stage in the ring
  static_assert(256 * kOutStride <= kBar, "the ring holds them");
  static_assert(kDynamic <= 232448, "shared memory of a block");
};

template <int D>
__global__ void __launch_bounds__(kPreThreads, 1)
prefix_attention_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ContTable ct,
                        const __grid_constant__ PagedAttnArgs a, int rows_per_tile, DeviceStatus* st) {
  using L = PreSmem<D>;
  // tensor memory: S of even tiles | S of odd tiles | O | P | Q
  constexpr uint32_t kTmemCols = 512, kO = 256, kP = 384, kQ = 448;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bar_full = base + L::kBar, bar_empty = bar_full + 8 * kPreRing, bar_q = bar_empty + 8 * kPreRing, bar_s = bar_q + 8,
                 bar_read = bar_s + 16, bar_p = bar_read + 16, bar_m = bar_p + 16, bar_o = bar_m + 16, bar_vfix = bar_o + 16;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + L::kMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + L::kMisc + 4);
  volatile float* max_s = reinterpret_cast<volatile float*>(base_ptr + L::kMax);
  volatile float* sum_s = reinterpret_cast<volatile float*>(base_ptr + L::kSum);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.H / a.Hkv;
  // which context, rows, head and piece: the row tiles of a piece stand side by side and find its keys in L2
  const int b = find_segment(ct.tile_cu, ct.n_req, (int)blockIdx.x);
  const int n_rt = (ct.max_rows[b] + rows_per_tile - 1) / rows_per_tile, at = (int)blockIdx.x - ct.tile_cu[b];
  const int rt = at % n_rt, hd = at / n_rt % a.Hkv, piece = at / (n_rt * a.Hkv);
  const int ctx_len = ct.ctx_len[b], n_tiles = (ctx_len + kPreTile - 1) / kPreTile;
  const int per = (n_tiles + ct.pieces[b] - 1) / ct.pieces[b], j0 = min(n_tiles, piece * per), n = min(n_tiles, j0 + per) - j0;
  const int token0 = (int)ct.tok_off[b] + j0 * kPreTile;
  const int x = (warp >> 2) & 1, t = (int)threadIdx.x & 127, t_local = t / G, head = hd * G + t - t_local * G;      // softmax threads: group, row, of it
  if (threadIdx.x == 256) {
    prefetch_tensormap(&tm_k); prefetch_tensormap(&tm_v);
    for (int s = 0; s < kPreRing; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
    mbar_init(bar_q, 256);
    for (int i = 0; i < 2; ++i) { mbar_init(bar_s + 8 * i, 1); mbar_init(bar_read + 8 * i, 128); mbar_init(bar_p + 8 * i, 128); mbar_init(bar_m + 8 * i, 128); mbar_init(bar_o + 8 * i, 1); }
    mbar_init(bar_vfix, 32);
    *abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == 9) { tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), kTmemCols); tmem_relinquish(); }
  // What a block needs first into L2 while the kernels in front finish (prefetches only: everything is read after the wait).  The rows are
  // guessed from the host's bounds: behind the first tiles of all blocks in HBM's queue, their loads took 3 to 5 us.
  if (warp < 8) {
    int before = 0;
    for (int i = 0; i < b; ++i) before += ct.max_rows[i];
    const long long guess = (long long)before + (long long)rt * rows_per_tile + t_local;
    if (x < L::kHalves && guess < a.n_rows && t_local < rows_per_tile) prefetch_l2(a.q + (guess * a.H + head) * D + x * 64);
    if (threadIdx.x == 0) { prefetch_l2(st); prefetch_l2(a.row_cu + ct.seq_cu[b]); prefetch_l2(a.row_cu + ct.seq_cu[b + 1]); }
  } else if (threadIdx.x == 256) {
    for (int u = 0; u < min(2 * n, kPreRing); ++u) {
      const PreLoad ld = prefix_load(u, n);
      tma_prefetch_5d(ld.v ? &tm_v : &tm_k, token0 + ld.tile * kPreTile, hd, 0);
    }
  }
  if (threadIdx.x < kPreTile) max_s[threadIdx.x] = kPreLowest;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  griddep_wait();
  griddep_launch();                                     // (behind the wait: the next kernel relies on what is in front of this one being complete)
  const int status = *reinterpret_cast<volatile int*>(&st->status);
  const long long row0 = a.row_cu[ct.seq_cu[b]], row1 = a.row_cu[ct.seq_cu[b + 1]];
  const long long first = row0 + (long long)rt * rows_per_tile;
  const bool refused = row0 < 0 || row1 > a.n_rows || row1 - row0 > ct.max_rows[b];       // more rows than the host's bounds: report, touch nothing
  if (refused || first >= row1 || status == RELAXKV_ERR_TIMEOUT) {
    if (refused && threadIdx.x == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_PREFIX_ATTN, (int)(row1 - row0), b);
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem_base, kTmemCols);
    return;
  }
  const int n_rows = (int)min((long long)rows_per_tile, row1 - first);
  const int tail = ctx_len % kPreTile;                  // tokens of the context's last tile, 0: all
  const bool fix_v = tail != 0 && j0 + n == n_tiles && n > 0;

  // Registers: 12 warps x 168 at launch = 8 x 224 + 4 x 56.
  if (warp >= 8) {
  reg_dealloc<56>();
  if (warp == 8) {
    // ================= TMA producer =================
    if (lane == 0) {
      for (int u = 0; u < 2 * n; ++u) {
        const int s = u % kPreRing;
        if (u >= kPreRing && !mbar_wait(bar_empty + 8 * s, (uint32_t)(u / kPreRing - 1) & 1, abort_flag)) break;
        mbar_expect_tx(bar_full + 8 * s, L::kTileBytes);
        const PreLoad ld = prefix_load(u, n);
        tma_load_5d(base + s * L::kTileBytes, ld.v ? &tm_v : &tm_k, bar_full + 8 * s, token0 + ld.tile * kPreTile, hd, 0);
      }
    }
    __syncwarp();
    if (fix_v) {
      // V rows behind the context belong to nobody (0 x NaN = NaN on the tensor core): zero them once their tile has landed
      const int u = 2 * n - 1, s = u % kPreRing;
      if (mbar_wait(bar_full + 8 * s, (uint32_t)(u / kPreRing) & 1, abort_flag)) {
        uint8_t* vt = base_ptr + s * L::kTileBytes;
        for (int i = lane; i < (kPreTile - tail) * 8 * L::kHalves; i += 32) {
          const int c = i & 7, r = tail + (i >> 3) % (kPreTile - tail), hf = (i >> 3) / (kPreTile - tail);
          *reinterpret_cast<uint4*>(vt + hf * L::kHalfBytes + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      mbar_arrive(bar_vfix);
    }
  } else if (warp == 9) {
    // ================= MMA issuer: the whole warp, one lane issues =================
    constexpr uint32_t idesc_qk = idesc_bf16_f32(kPreTile, kPreTile, 0), idesc_pv = idesc_bf16_f32(kPreTile, D, 1);
    constexpr uint32_t hi = desc_hi_sw128(1024);
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity & 1u, abort_flag)); };
    // number, buffer and phase of the next load, which is always the next to be used; a buffer that no later tile takes is not reported free (an
    // arrival that nobody waits for could come when the block has gone)
    int at_u = 0, s = 0;
    uint32_t phase = 0;
    auto step = [&]() { ++at_u; if (++s == kPreRing) { s = 0; phase ^= 1u; } };
    auto issue_qk = [&](int j) -> bool {                // S_j = Q K_j^T
      if (!wait(bar_full + 8 * s, phase)) return false;
      if (j > 1 && !wait(bar_read + 8 * (j & 1), (uint32_t)((j >> 1) - 1))) return false;         // S_{j-2} is in registers
      tc_fence_after();
      warp_mma_ts_kmajor<L::kHalves>(tmem_base + (j & 1) * 128, tmem_base + kQ, desc_lo(base + s * L::kTileBytes, 16), hi, idesc_qk);
      if (at_u + kPreRing < 2 * n) warp_mma_commit(bar_empty + 8 * s);
      warp_mma_commit(bar_s + 8 * (j & 1));
      step();
      return true;
    };
    bool ok = n > 0 && wait(bar_q, 0);
    for (int j = 0; ok && j < min(n, 2); ++j) ok = issue_qk(j);
    for (int j = 0; ok && j < n; ++j) {
      if (j + 2 < n && !(ok = issue_qk(j + 2))) break;
      if (!(ok = wait(bar_full + 8 * s, phase))) break;
      if (fix_v && j == n - 1 && !(ok = wait(bar_vfix, 0))) break;
      if (!(ok = wait(bar_p + 8 * (j & 1), (uint32_t)(j >> 1)))) break;
      tc_fence_after();
      warp_mma_ts_mnmajor(tmem_base + kO, tmem_base + kP, desc_lo(base + s * L::kTileBytes, L::kHalfBytes), hi, idesc_pv, j > 0 ? 1u : 0u);
      if (at_u + kPreRing < 2 * n) warp_mma_commit(bar_empty + 8 * s);
      warp_mma_commit(bar_o + 8 * (j & 1));
      step();
    }
  }
  } else {
    reg_alloc<224>();
    // ================= softmax: thread = (row of the step, head) = TMEM lane; x: even or odd tiles =================
    const bool mine = t_local < n_rows;
    const long long row = first + t_local;
    const uint32_t lane_base = tmem_base + ((uint32_t)((warp & 3) * 32) << 16), t_s = lane_base + x * 128, t_o = lane_base + kO;
    if (x < L::kHalves) {                               // of Q, each group brings 64 dims
      uint32_t w[32];
      const uint4* q = reinterpret_cast<const uint4*>(a.q + (row * a.H + head) * D + x * 64);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 v = mine ? q[c] : make_uint4(0, 0, 0, 0);
        w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
      }
      tmem_st32(lane_base + kQ + x * 32, w);
      tmem_wait_st();
      tc_fence_before();
    }
    mbar_arrive(bar_q);
    const bool busy = __any_sync(0xffffffffu, mine);    // a warp without rows only keeps step
    float m = kPreLowest, z = 0.f;                      // the row's maximum when this group last saw it, the group's sum relative to that
    bool ok = true;
    for (int j = x; j < n; j += 2) {
      ok = mbar_wait(bar_s + 8 * x, (uint32_t)(j >> 1) & 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      if (!busy) {                                      // (a warp that ran ahead would arrive twice in one phase of a barrier)
        mbar_arrive(bar_read + 8 * x);
        if (j > 0) ok = mbar_wait(bar_m + 8 * (x ^ 1), (uint32_t)((j - 1) >> 1) & 1, abort_flag);
        if (ok) mbar_arrive(bar_m + 8 * x);
        if (ok && j > 0) ok = mbar_wait(bar_o + 8 * (x ^ 1), (uint32_t)((j - 1) >> 1) & 1, abort_flag);
        if (ok) mbar_arrive(bar_p + 8 * x);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        continue;
      }
      uint32_t s[kPreTile];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(t_s + c * 32, &s[c * 32]);
      tmem_wait_ld();
      tc_fence_before();
      mbar_arrive(bar_read + 8 * x);
      const int limit = ctx_len - (j0 + j) * kPreTile;
      if (limit < kPreTile) {
#pragma unroll
        for (int i = 0; i < kPreTile; ++i)
          if (i >= limit) s[i] = 0xff800000u;           // -inf
      }
      float mx[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) mx[e] = fmaxf(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1]));
#pragma unroll
      for (int i = 16; i < kPreTile; i += 2) mx[(i >> 1) & 7] = fmax3(mx[(i >> 1) & 7], __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
      const float m_tile = fmax3(fmax3(mx[0], mx[1], mx[2]), fmax3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * a.scale_log2;
      float scale = a.scale_log2;
      if (__any_sync(0xffffffffu, fabsf(m_tile) > kPreExact)) {
#pragma unroll
        for (int i = 0; i < kPreTile; ++i) s[i] = __float_as_uint(__uint_as_float(s[i]) * scale);
        scale = 1.f;
      }
      if (j > 0) {                                      // the other group's maximum of the tile before
        ok = mbar_wait(bar_m + 8 * (x ^ 1), (uint32_t)((j - 1) >> 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
      }
      const float m_old = max_s[t];
      const bool need = m_tile > m_old + kPreRescale;
      const float m_new = need ? m_tile : m_old;
      if (need) max_s[t] = m_new;
      mbar_arrive(bar_m + 8 * x);
      z *= fast_exp2(m - m_new);                        // (1 as long as nothing has changed)
      m = m_new;
      uint32_t pk[64];
      z += prefix_exponentials(s, pk, scale, -m);
      if (j > 0) {                                      // O of the tile before is complete, its P is not needed any more
        ok = mbar_wait(bar_o + 8 * (x ^ 1), (uint32_t)((j - 1) >> 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        if (__any_sync(0xffffffffu, need)) {
          const float alpha = fast_exp2(m_old - m_new);
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
      }
      tmem_st32(lane_base + kP, pk);
      tmem_st32(lane_base + kP + 32, pk + 32);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(bar_p + 8 * x);
    }
    // ---- the output, each thread half the dims of its row ----
    if (ok && n > 0) ok = mbar_wait(bar_o, (uint32_t)((n - 1) >> 1) & 1, abort_flag);
    if (ok && n > 1) ok = mbar_wait(bar_o + 8, (uint32_t)((n - 2) >> 1) & 1, abort_flag);
    const float m_end = ok ? max_s[t] : m;
    sum_s[x * kPreTile + t] = z * fast_exp2(m - m_end);
    asm volatile("bar.sync 1, 256;" ::: "memory");
    ok = __all_sync(0xffffffffu, ok && !*abort_flag);
    tc_fence_after();
    if (ok && busy) {
      const float zz = sum_s[t] + sum_s[kPreTile + t];
      const bool none = zz == 0.f;                      // no key, or none of a logit above -inf (NaN stays NaN)
      const float inv = none ? 0.f : 1.f / zz, lse = none ? -INFINITY : (m_end + log2f(zz)) * kLn2Pre;
      const bool direct = a.n_slots == 1;
      const bool store = mine && (!direct || check_row(a, ct, row, x == 0, st).seq >= 0);
      const long long slot = ((long long)piece * a.n_rows + row) * a.H + head;
      uint8_t* stage = base_ptr + threadIdx.x * L::kOutStride;        // (all tiles have been consumed)
#pragma unroll 1
      for (int c = 0; c < D / 64; ++c) {
        uint32_t o[32];
        if (n > 0) { tmem_ld32(t_o + x * (D / 2) + c * 32, o); tmem_wait_ld(); }
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = none ? 0u : __float_as_uint(__uint_as_float(o[i]) * inv);
        if (!direct) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(stage + c * 128 + i * 4) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        } else if (store) {
          uint16_t* p = a.out + (row * a.H + head) * D + x * (D / 2) + c * 32;
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
        }
      }
      if (!direct && store) {                           // a row's half as one copy out of shared memory
        fence_proxy_async_smem();
        bulk_store(a.part_o + slot * D + x * (D / 2), smem_u32(stage), D * 2);
        if (x == 0) a.part_lse[slot] = lse;
        bulk_store_commit_and_drain();
      }
      if (store && x == 0 && direct && a.lse_out) a.lse_out[(long long)head * a.n_rows + row] = lse;
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
  if (warp == 9) { tc_fence_after(); tmem_dealloc(tmem_base, kTmemCols); }
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
                                            const relaxkv_continuation_rows* rows, const void* q, void* out, float* lse_out,
                                            void* workspace, size_t workspace_bytes, ContTable& ct, PagedAttnArgs& a) {
  relaxkv_status rc = check_contexts(shape);
  if (rc != RELAXKV_OK) return rc;
  bool any_ctx = false;
  for (int b = 0; b < shape->n_req; ++b) any_ctx |= shape->h_ctx_len[b] > 0;
  if (any_ctx && (rc = check_cache(shape, cache, true)) != RELAXKV_OK) return rc;
  fill_contexts(ct, shape, any_ctx ? cache : nullptr, 0);
  for (int b = 0; b < ct.n_req; ++b)
    if (ct.ctx_len[b] > 0 && ct.tok_off[b] > kContTokensMost - ct.ctx_len[b]) return RELAXKV_ERR_UNSUPPORTED_SHAPE;      // a tile's place is 32 bits
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
  relaxkv_status rc = prepare_continuations(shape, cache, store, rows, q, out, lse_out, workspace, workspace_bytes, ct, a);
  if (rc != RELAXKV_OK || rows->n_rows == 0) return rc;
  const int sms = sm_count_of_current_device();
  if (sms <= 0) return RELAXKV_ERR_CUDA;
  const int D = shape->head_dim, rows_per_tile = kPreTile / (a.H / a.Hkv), slots = cont_slots(a.n_rows);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // ---- few rows and short contexts: one launch, each row by itself ----
  // One cluster per (row, KV head), all at once and twelve tiles to a block at most: the launches are what such a call takes.  One and four rows of 32 / 8
  // heads over 3 K tokens 10.7 and 11.8 us (14.2 and 14.7 the other way), 6 K 14.2 and 16.6 (15.5 and 19.5), 10 K 19.5 and 23.0 (18.8 and 21.3); eight
  // rows over 3 K, not all at once, 22.8 (18.7).
  int longest = 0;
  for (int b = 0; b < ct.n_req; ++b)
    if (ct.max_rows[b] > 0) longest = std::max(longest, ct.ctx_len[b]);
  const long long all_tiles = ((long long)longest + 63) / 64 + (a.max_len + 63) / 64;
  if (a.n_rows * a.Hkv * kPagCluster <= 2LL * sms && all_tiles <= 12 * kPagCluster) {
    a.ctx_keys = longest > 0 ? CTX_KEYS_ALL : CTX_KEYS_NONE;
    a.ctx_block = 64;
    a.n_splits = cluster_that_fits(shape, (int)std::max<long long>(1, std::min<long long>(kPagCluster, all_tiles / 2)), a.n_rows * a.Hkv);
    a.cluster = a.n_splits > 1;
    a.n_slots = 1;
    return launch_paged_attention(shape, cache, store, ct, a, s);
  }
  // ---- pieces of the rows' own keys (0: there are none), and of the contexts ----
  const bool own = a.max_len > 0;
  // Up to eight pieces of a row's own keys are a cluster that merges them and the pieces of its context, too; more go through slots and the
  // merge behind.
  const long long own_tiles = ((long long)a.max_len + 63) / 64;
  a.n_splits = own ? cluster_that_fits(shape, paged_cluster(a.n_rows * a.Hkv, own_tiles, sms, kPagCluster), a.n_rows * a.Hkv) : 0;
  a.cluster = a.n_splits > 0;
  const int own_pieces = !own || a.cluster ? 0 : paged_pieces(a.n_rows * a.Hkv, own_tiles, sms, std::max(1, slots / 4));
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
  a.slot0 = own_pieces > 0 ? most : kContSlotsMost;     // without such pieces no slot is theirs
  a.n_slots = most + own_pieces;
  if (own_pieces > 0) a.n_splits = own_pieces;
  if (a.cluster && most == 0 && a.n_splits == 1) {      // nothing to merge
    a.cluster = 0;
    a.n_slots = 1;
  }
  if (a.cluster && a.n_slots == 1) a.n_slots = 2;       // (the prefix kernel is not the last)
  if (a.n_slots <= 1 && !all) a.n_slots = 2;            // rows without any key: the merge writes their zeros
  if (most > 0) {
    rc = D == 128 ? launch_prefix<128>(cache, ct, a, rows_per_tile, s) : launch_prefix<64>(cache, ct, a, rows_per_tile, s);
    if (rc != RELAXKV_OK) return rc;
  }
  a.behind_prefix = most > 0;
  if (own && (rc = launch_paged_attention(shape, cache, store, ct, a, s)) != RELAXKV_OK) return rc;
  return a.n_slots == 1 || a.cluster ? RELAXKV_OK : launch_continuation_merge(ct, a, D, s);
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
  relaxkv_status rc = prepare_continuations(shape, cache, store, rows, q, out, lse_out, workspace, workspace_bytes, ct, a);
  if (rc != RELAXKV_OK) return rc;
  if (n_select > 0x7fffffff / block_size) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (rows->n_rows == 0) return RELAXKV_OK;
  const int sms = sm_count_of_current_device();
  if (sms <= 0) return RELAXKV_ERR_CUDA;
  bool any_ctx = false;
  for (int b = 0; b < ct.n_req; ++b) any_ctx |= ct.ctx_len[b] > 0;
  a.ctx_keys = any_ctx ? CTX_KEYS_LISTED : CTX_KEYS_NONE;
  a.lists = blocks; a.n_select = n_select; a.ctx_block = block_size;
  for (int b = 0; b < ct.n_req; ++b)
    if (ct.max_rows[b] > 0) a.listed_most = std::max(a.listed_most, (int)std::min<long long>(n_select, ((long long)ct.ctx_len[b] + block_size - 1) / block_size));
  const long long tiles = ((long long)a.listed_most * block_size + 63) / 64 + (a.max_len + 63) / 64;
  a.n_splits = cluster_that_fits(shape, paged_cluster(a.n_rows * a.Hkv, tiles, sms, kPagCluster), a.n_rows * a.Hkv);
  a.cluster = a.n_splits > 1;
  if (a.n_splits == 0) a.n_splits = paged_pieces(a.n_rows * a.Hkv, tiles, sms, cont_slots(a.n_rows));
  a.slot0 = 0;
  a.n_slots = a.cluster ? 1 : a.n_splits;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((rc = launch_paged_attention(shape, cache, store, ct, a, s)) != RELAXKV_OK) return rc;
  return a.n_slots == 1 ? RELAXKV_OK : launch_continuation_merge(ct, a, shape->head_dim, s);
}
