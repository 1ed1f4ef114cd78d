// Attention of many rows of a sequence over its tokens in the 8-bit store: a question, a long draft (relaxkv_quantized_attention).
//
// Rows x heads of a group meet the same keys, so they are the rows of a matrix product: a block owns 128 of them (128 / G rows of
// one sequence), one KV head and a run of 128-token tiles.  Eight warps bring a tile, four its K and four its V: 8-bit values out
// of the pages in 16-byte pieces, two tiles ahead, made fp16, exactly, and written where the tensor cores read them (K as rows of
// dims, V as rows of the contraction, 128-byte swizzle).  S = Q K^T with Q in tensor memory as fp16 (exactly, times a power of two
// per row); a thread makes weights of a row of S, which take its place as fp16; O += P V.  The exponents of the keys go on the
// scores, those of the values on the weights, relative to the largest so far of the tokens that a row sees: p = 2^(s - m + 11 + e_t
// - E). Two groups of four warps take the even and the odd tiles: the weights of one tile are made while the products of the other
// run.  S of tile j + 2 is made when P of tile j has been used; a group hands its P over when O of the tile before is complete,
// which is also when O may be rescaled; a row's running maximum goes from group to group through shared memory, sums stay with the
// groups.  K is written a tile ahead of V, or the weights of a tile wait for a value tile that waits for them. Every wait is
// bounded.
//
// Measured (int8, D 128): 57 rows of 40 / 8 heads over 16 K 62.9 us (the products alone, at 1.66 PFLOP/s, 11.5; the kernel of few
// rows 123).  Bound by issue, not by the tensor cores (21 % of the time) or memory: a tile's 128 x 128 weights and its two
// conversions to fp16 are some 2100 instructions of each of the SM's four schedulers, which five warps each (two of rows, one each
// of K and V, the products') issue at half their rate, 4200 clk a tile.  No faster, at 62.7 us then: weights in one pass with a
// reference that is a whole number (62.7), exponents within the fp16 tiles in place of factors on scores and weights (65.4: the
// conversions get longer), both groups on halves of the same tile (68.4: all wait and all take exponentials at once), 144 or 128
// registers for the rows' threads (62.9). Weighing the last tile of a row relative to what the row sees of it took 1 us.
#include "quantized_attention.cuh"
#include <atomic>

namespace relaxkv {

using namespace ptx;

constexpr int kQrTile = 128, kQrThreads = 640;           // tokens of a tile; warps 0-3 and 4-7: a row per thread, 8-11: K, 12-15: V, 16: products, three idle
constexpr float kQrShift = 11.f, kQrGrow = 4.f;          // weights begin at 2^11 and are rescaled when a row's maximum grew by 2^4
// Factors of keys are up to 2^90, what is above that of a tile's largest goes to the rows' scales: a product of Q and key values (2^31 at most) stays within fp32 before its row's scale.
constexpr int kQrKeyMost = 90;
// Values' factors are relative to the largest exponent so far, a second set to one 2^120 below: for rows that do not see tokens whose exponents are more than 100 above what they see.
constexpr int kQrBelow = 120, kQrNear = 100;
constexpr float kQrExact = 32768.f;                      // logits (in log2 units) up to this are not rounded by themselves: 2^-9 of a weight
using QrWalk = Walk<kQrTile, 4, 2, 128>;                 // a task's start and end take as long as four tiles (57 rows over 16 K: of two 68 us, of three to six 64)

template <int D>
struct QrSmem {
  static constexpr int kHalves = D / 64, kHalfBytes = kQrTile * 128, kTileBytes = kHalves * kHalfBytes;
  static constexpr int kV = 2 * kTileBytes;              // K[2] | V[2]
  static constexpr int kScale = 4 * kTileBytes;          // of the last four tiles: factors of the keys' scores, of the values' weights, these 2^kQrBelow times as large
  static constexpr int kRaw = kScale + 4 * 3 * kQrTile * 4;      // 8-bit values of two tiles as they come, K and V: every piece is one thread's
  static constexpr int kRawTile = 2 * kQrTile * D;
  static constexpr int kBar = kRaw + 2 * kRawTile;
  // full_k[2], full_v[2], empty_k[2], empty_v[2], s[2], m[2], o[2], scale[4], p, q: those of two or four belong to every second or fourth tile, so that nobody who
  // waits for one phase can be two behind
  static constexpr int kNumBars = 20;
  static constexpr int kMax = kBar + 8 * kNumBars + 8;   // running maximum of every row; its sums, by group
  static constexpr int kTotal = kMax + 3 * 4 * kQrRows;
  static constexpr int kDynamic = kTotal + 1024;
  static_assert(kDynamic <= 232448 - 1024, "shared memory of a block");
};

// f16 x f16 -> fp32, A K-major.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int m, int n, int b_mn_major) {
  return (1u << 4) | (static_cast<uint32_t>(b_mn_major) << 16) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24);
}

// Sixteen 8-bit values as fp16, in their order.
template <int TYPE>
__device__ __forceinline__ void to_half_16(const uint4& r, uint4* out) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TYPE == RELAXKV_INT8) {
      const uint32_t b = w[i] ^ 0x80808080u;
      h[2 * i] = int8_to_half2<0x4140>(b); h[2 * i + 1] = int8_to_half2<0x4342>(b);
    } else { h[2 * i] = e4m3_to_half2(w[i], 0); h[2 * i + 1] = e4m3_to_half2(w[i], 1); }
  }
  out[0] = make_uint4(h[0], h[1], h[2], h[3]);
  out[1] = make_uint4(h[4], h[5], h[6], h[7]);
}

// A barrier of some of the warps at which they also agree whether to go on: none waits for one that has left after a wait that ran out.
template <int ID, int THREADS>
__device__ __forceinline__ bool meet(bool ok) {
  int all;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, %3, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
               : "=r"(all) : "r"((int)ok), "n"(ID), "n"(THREADS) : "memory");
  return all != 0;
}

template <int D, int TYPE>
__global__ void __launch_bounds__(kQrThreads, 1)
quantized_rows_kernel(const __grid_constant__ QuantAttnArgs a, DeviceStatus* st) {
  using L = QrSmem<D>;
  constexpr uint32_t kTmemCols = 512, kO = 256, kQ = 384;      // tensor memory: S, then P, of even tiles | of odd tiles | O | Q
  extern __shared__ uint8_t smem_raw[];
  __shared__ QrWalk::Shared walk_s;
  __shared__ volatile uint32_t tmem_slot;
  __shared__ volatile int abort_s;
  __shared__ int largest_s[2][4], e_s[8];                 // largest exponents of the values: of each of the four warps' tokens; up to the last eight tiles
  __shared__ int largest_k_s[2][4], over_s[4];            // of the keys: of each warp's tokens; by how much the last four tiles' are above kQrKeyMost
  __shared__ uint32_t top_s[2][kQrRows];                 // largest bits of a row's dims, by half
  __shared__ int e_part_s[kQrRows];                       // what O of a row is relative to that does not see the last tile, or not all of it
  __shared__ uint32_t gone_s[4][4], nan_s[4][4];          // tokens of the last four tiles whose blocks do not exist; whose values are NaN
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t full_k = base + L::kBar, full_v = full_k + 16, empty_k = full_v + 16, empty_v = empty_k + 16, bar_s = empty_v + 16, bar_m = bar_s + 16,
                 bar_o = bar_m + 16, bar_scale = bar_o + 16, bar_p = bar_scale + 32, bar_q = bar_p + 8;
  volatile int* abort_flag = &abort_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(full_k + 8 * i, 128); mbar_init(full_v + 8 * i, 128); mbar_init(empty_k + 8 * i, 1); mbar_init(empty_v + 8 * i, 1);
      mbar_init(bar_s + 8 * i, 1); mbar_init(bar_m + 8 * i, 128); mbar_init(bar_o + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(bar_scale + 8 * i, 128);
    mbar_init(bar_p, 128); mbar_init(bar_q, 256);
    abort_s = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
  }
  if (warp == 16) { tmem_alloc(smem_u32(const_cast<uint32_t*>(&tmem_slot)), kTmemCols); tmem_relinquish(); }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  griddep_launch();                                      // (behind the allocation: the join's blocks take none)
  griddep_wait();
  QrWalk g;
  const bool any = g.begin(a, walk_s, st);
  const int status = *reinterpret_cast<volatile int*>(&st->status);
  if (!any || status == RELAXKV_ERR_TIMEOUT) {
    if (tid == 0) a.chain[blockIdx.x].c0 = -1;
    __syncthreads();
    if (warp == 16) tmem_dealloc(tmem_base, kTmemCols);
    return;
  }
  const int G = a.G, rpt = a.rows_per_tile, bs_mask = (1 << a.block_shift) - 1;

  // Registers: 20 warps x 96 at launch = 8 x 136 + 8 x 80 + 4 x 48.
  if (warp < 8) {
    reg_alloc<136>();
    // ================= weights: thread = (row of the sequence, head) = lane of tensor memory; x: even or odd tiles =================
    const int x = warp >> 2, t = tid & 127, t_local = t / G, in_group = t - t_local * G;
    const uint32_t lane_base = tmem_base + ((uint32_t)((warp & 3) * 32) << 16), t_s = lane_base + x * 128, t_o = lane_base + kO;
    volatile float* max_s = reinterpret_cast<volatile float*>(base_ptr + L::kMax);
    volatile float* sum_s = max_s + kQrRows;
    bool ok = true;
    uint32_t jj = 0;                                     // tiles so far, over all tasks
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity & 1u, abort_flag)); };
    for (bool more = true; more && ok;) {
      const long long row = (long long)g.s.first + (long long)g.tile * rpt + t_local;
      const int head = g.hd * G + in_group;
      const bool exists = t_local < min(rpt, g.s.n - g.tile * rpt);
      const int seen = exists ? row_tokens(a, g.seq, g.s, row, x == 0 && in_group == 0 && g.hd == 0 && g.j0 == 0, st) : -1;
      // ---- Q: as fp16 times 2^-exponent, two dims to a word; each group brings half of them, and both know the largest ----
      // A row that is no number meets the keys as zeros, so that what it does not see weighs nothing; its result becomes NaN at the end, where it has seen a token.
      int qe;                                            // exponent of the row's scale
      bool finite;
      {
        uint32_t w[D / 4], top = 0;
        const uint4* q = reinterpret_cast<const uint4*>(a.q + (row * a.H + head) * D) + x * (D / 16);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          const uint4 v = exists ? q[c] : make_uint4(0, 0, 0, 0);
          w[4 * c] = v.x; w[4 * c + 1] = v.y; w[4 * c + 2] = v.z; w[4 * c + 3] = v.w;
        }
#pragma unroll
        for (int c = 0; c < D / 4; ++c) top = __vmaxu2(top, w[c] & 0x7fff7fffu);
        top = max(top & 0xffffu, top >> 16);
        top_s[x][t] = top;
        if (!(ok = meet<2, 256>(ok))) break;
        top = max(top, top_s[x ^ 1][t]);
        finite = top < 0x7f80u;
        const int e = max((int)(top >> 7) - 127 - 14, -120);
        const float inv = __uint_as_float((uint32_t)(127 - (finite ? e : 0)) << 23);
#pragma unroll
        for (int c = 0; c < D / 4; ++c) {
          const __half2 y = __floats2half2_rn(__uint_as_float(w[c] << 16) * inv, __uint_as_float(w[c] & 0xffff0000u) * inv);
          w[c] = finite ? *reinterpret_cast<const uint32_t*>(&y) : 0u;
        }
        qe = finite && top != 0 ? e : 0;                 // (zeros are zeros by any scale)
        if constexpr (D == 128) tmem_st32(lane_base + kQ + 32 * x, w); else tmem_st16(lane_base + kQ + 16 * x, w);
        tmem_wait_st();
        tc_fence_before();
      }
      mbar_arrive(bar_q);
      const bool busy = __any_sync(0xffffffffu, seen >= 0);          // a warp without rows only keeps step
      const int n = g.j1 - g.j0;
      const uint32_t jj0 = jj;
      float m = kNothing, z = 0.f;                       // the row's maximum when this group last saw it, the group's sum relative to that
      for (int i = (int)((jj0 ^ x) & 1); i < n; i += 2) {
        jj = jj0 + i;
        const int j = g.j0 + i, ring = jj & 3;
        if (!(ok = wait(bar_scale + 8 * ring, jj >> 2)) || !(ok = wait(bar_s + 8 * x, jj >> 1))) break;
        tc_fence_after();
        if (!busy) {
          if (jj > 0 && !(ok = wait(bar_m + 8 * (x ^ 1), (jj - 1) >> 1))) break;
          mbar_arrive(bar_m + 8 * x);
          if (jj > 0 && !(ok = wait(bar_o + 8 * (x ^ 1), (jj - 1) >> 1))) break;
          mbar_arrive(bar_p);
          continue;
        }
        const float* ks = reinterpret_cast<const float*>(base_ptr + L::kScale) + ring * 3 * kQrTile;
        const float* vs = ks + kQrTile;
        const int limit = seen < 0 ? kQrTile : seen - j * kQrTile;      // (rows that are not written see all: nothing to hide costs half as much)
        const bool slow = __any_sync(0xffffffffu, limit < kQrTile || (gone_s[ring][0] | gone_s[ring][1] | gone_s[ring][2] | gone_s[ring][3]) != 0);
        const bool factors = slow && (nan_s[ring][0] | nan_s[ring][1] | nan_s[ring][2] | nan_s[ring][3]) != 0;
        // (never 0: what is not seen stays -inf)
        const float qs = fmaxf(__uint_as_float((uint32_t)(127 + min(qe + over_s[ring], 127)) << 23) * a.scale_log2, 1.4e-45f);
        // 32 scores times their keys' scales; what the row does not see (its tokens from `limit` on, tokens without a block) becomes -inf
        auto scores = [&](int c, float* y) -> uint32_t {
          uint32_t w[32];
          tmem_ld32(t_s + c * 32, w);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 k4 = *reinterpret_cast<const float4*>(ks + c * 32 + e);
            mul2(y[e], y[e + 1], __uint_as_float(w[e]), __uint_as_float(w[e + 1]), k4.x, k4.y);
            mul2(y[e + 2], y[e + 3], __uint_as_float(w[e + 2]), __uint_as_float(w[e + 3]), k4.z, k4.w);
          }
          uint32_t hidden = 0;
          if (slow) {
            hidden = (limit >= 32 * (c + 1) ? 0u : limit <= 32 * c ? 0xffffffffu : 0xffffffffu << (limit - 32 * c)) | gone_s[ring][c];
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (hidden >> e & 1) y[e] = -INFINITY;
          }
          return hidden;
        };
        // (chunk by chunk: unrolled over the tile, the code of a warp that has its scheduler almost for itself came from far, 16 K clk a tile)
        float top = kNothing;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float y[32], mx[4];
          scores(c, y);
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(y[2 * e], y[2 * e + 1]);
#pragma unroll
          for (int e = 8; e < 32; e += 2) mx[(e >> 1) & 3] = fmax3(mx[(e >> 1) & 3], y[e], y[e + 1]);
          top = fmax3(top, fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        }
        if (jj > 0 && !(ok = wait(bar_m + 8 * (x ^ 1), (jj - 1) >> 1))) break;      // the other group's maximum of the tile before
        const float m_tile = top * qs;                   // (qs > 0)
        float m_old = kNothing;
        if (i > 0) m_old = max_s[t];
        const bool grows = m_tile > m_old + kQrGrow;
        const float m_new = grows ? m_tile : m_old;
        max_s[t] = m_new;
        mbar_arrive(bar_m + 8 * x);
        z *= fast_exp2(m - m_new);
        m = m_new;
        // The values' exponents are weighed relative to the largest so far of the tokens that the row sees: of the last tile that it sees, when that is a part of it, the part's largest,
        // e_less below the tile's.  The weights of that tile grow by as much (2^e_grow with the factors that they meet), and their sum comes down again.
        const bool cut = limit > 0 && limit < kQrTile;
        int e_less = 0, e_grow = 0;
        bool second = false;
        // (only where the tile has a larger one than all before it)
        if (slow && __any_sync(0xffffffffu, cut) && (i == 0 || e_s[jj & 7] != e_s[(jj - 1) & 7])) {
          // a value's exponent, less that of the tile, + kQrShift + 127: from its factor, or from the second one where that is 0
          auto exponent = [&](int at) -> int {
            const int f = (int)(__float_as_uint(vs[at]) >> 23);
            if (f == 255) return -1000;                  // (NaN)
            return f > 0 ? f : (int)(__float_as_uint(vs[at + kQrTile]) >> 23) - kQrBelow;      // (none: far below)
          };
          int upto = -1000;                              // of tokens up to 4 lane + 3
#pragma unroll 1
          for (int b = 0; b < 4; ++b) upto = max(upto, exponent(4 * lane + b));
#pragma unroll 1
          for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto = max(upto, y);
          }
          const int some = min(max(limit, 0), kQrTile - 1), words = some >> 2;
          int most = __shfl_sync(0xffffffffu, upto, max(words - 1, 0));
          if (words == 0) most = -1000;
#pragma unroll 1
          for (int b = 0; b < (some & 3); ++b) most = max(most, exponent(4 * words + b));
          most -= (int)kQrShift + 127;
          const int e_tile = e_s[jj & 7], e_before = i > 0 ? e_s[(jj - 1) & 7] : kExpLeast;       // (a row that sees some of it has seen all of the tiles before)
          if (cut) e_less = e_tile - max(e_before, e_tile + most);
          e_grow = e_less > kQrNear ? e_less - kQrBelow : e_less;
          if (e_less > kQrNear) vs += kQrTile;
          second = __any_sync(0xffffffffu, e_less > kQrNear);
        }
        const float m_less = m - (float)e_grow;
        // s * qs - m in one rounding keeps what the rounding of m has cut off: the same factor on all weights of the row, which their sum takes out again; very large logits are
        // rounded first, or the factor would leave the range of fp16
        const bool large = __any_sync(0xffffffffu, fabsf(m_tile) > kQrExact);
        const float q2 = large ? 1.f : qs;
        float z0 = 0.f, z1 = 0.f, z2 = 0.f, z3 = 0.f;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float y[32];
          uint32_t pk[16];
          const uint32_t hidden = scores(c, y);
          if (large) {
#pragma unroll
            for (int e = 0; e < 32; ++e) y[e] *= qs;
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            float p[4];
            const float4 v4 = *reinterpret_cast<const float4*>(vs + c * 32 + e);
            fma2(p[0], p[1], y[e], y[e + 1], q2, q2, -m_less, -m_less);
            fma2(p[2], p[3], y[e + 2], y[e + 3], q2, q2, -m_less, -m_less);
#pragma unroll
            for (int u = 0; u < 4; ++u) p[u] = fast_exp2(p[u]);
            add2(z0, z1, p[0], p[1]);
            add2(z2, z3, p[2], p[3]);
            mul2(p[0], p[1], p[0], p[1], v4.x, v4.y);
            mul2(p[2], p[3], p[2], p[3], v4.z, v4.w);
#pragma unroll
            for (int u = 0; u < 4; u += 2) {
              const __half2 h = __floats2half2_rn(p[u], p[u + 1]);
              pk[(e + u) >> 1] = *reinterpret_cast<const uint32_t*>(&h);
            }
          }
          if (factors || second) {                       // what is not seen weighs nothing, whatever its factor
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (hidden >> e & 1) pk[e >> 1] &= e & 1 ? 0x0000ffffu : 0xffff0000u;
          }
          tmem_st16(t_s + c * 16, pk);                   // (where scores were that have been read)
        }
        z = fmaf((z0 + z1) + (z2 + z3), __uint_as_float((uint32_t)(127 - e_grow) << 23), z);
        if (jj > 0) {                                    // O of the tile before is complete
          if (!(ok = wait(bar_o + 8 * (x ^ 1), (jj - 1) >> 1))) break;
          tc_fence_after();
        }
        int e_up = i > 0 ? e_s[jj & 7] - e_s[(jj - 1) & 7] : 0;
        if (slow) {
          if (limit >= 0 && limit < kQrTile) e_part_s[t] = cut ? e_s[jj & 7] - e_less : e_s[(jj - 1) & 7];      // (of the last tile that the row sees)
          e_up = cut ? e_up - e_less : limit > 0 ? e_up : 0;
        }
        if (i > 0 && __any_sync(0xffffffffu, grows || e_up != 0)) {
          const float alpha = fast_exp2(m_old - m_new - (float)e_up);
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld32(t_o + c * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            tmem_st32(t_o + c * 32, o);
          }
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(bar_p);
      }
      // ---- the results, each group half the dims ----
      jj = jj0 + n;
      if (ok && jj > 1) ok = wait(bar_o + 8 * (jj & 1), (jj - 2) >> 1);
      if (ok) ok = wait(bar_o + 8 * (~jj & 1), (jj - 1) >> 1);
      const float m_end = max_s[t];                      // (of a warp without rows: anything)
      sum_s[x * kQrRows + t] = z * fast_exp2(m - m_end);
      ok = meet<2, 256>(ok && !*abort_flag);
      const int e_last = seen >= 0 && seen < (long long)g.j1 * kQrTile ? e_part_s[t] : e_s[(jj - 1) & 7];      // (of a row that has seen no token: anything)
      const bool whole = g.whole();
      const int slot = g.slot();
      if (tid == 0) {
        Chain* c = a.chain + blockIdx.x;                 // (the last task's stays)
        int c0 = -1, c1 = 0;
        if (g.j1 < g.tiles) g.blocks_of(&c0, &c1);
        c->c0 = c0; c->c1 = c1; c->row = g.s.first + g.tile * rpt; c->head = g.hd; c->cols = min(rpt, g.s.n - g.tile * rpt) * G;
      }
      const uint32_t live = __ballot_sync(0xffffffffu, seen >= 0);
      if (x == 0 && lane == 0) a.chain[blockIdx.x].live[warp] = live;
      if (ok && busy) {
        tc_fence_after();
        const float zz = sum_s[t] + sum_s[kQrRows + t];
        const bool none = zz == 0.f;                     // no token, or none of a logit above -inf (NaN stays NaN)
        const float nan = __uint_as_float(0x7fc00000u);
        const float inv = none ? 0.f : finite ? one_over(zz * 2048.f) : nan, grow = __uint_as_float((uint32_t)(e_last + 127) << 23);
        static_assert(kQrShift == 11.f, "2^11");
        const float lse2 = none ? -INFINITY : finite ? m_end + log2_of(zz) : nan;
#pragma unroll 1
        for (int c = x * (D / 64); c < (x + 1) * (D / 64); ++c) {
          uint32_t o[32];
          tmem_ld32(t_o + c * 32, o);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = none ? 0u : __float_as_uint(__uint_as_float(o[e]) * inv * grow);
          if (seen >= 0 && !whole) {
            float* p = a.part_o + ((long long)slot * kQrRows + t) * D + c * 32;
#pragma unroll
            for (int e = 0; e < 32; e += 8) st_global_32b(p + e, o + e);
          } else if (seen >= 0) {
            uint16_t* p = a.out + (row * a.H + head) * D + c * 32;
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              uint32_t w[4];
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const __nv_bfloat162 h2 = __floats2bfloat162_rn(__uint_as_float(o[e + 2 * u]), __uint_as_float(o[e + 2 * u + 1]));
                w[u] = *reinterpret_cast<const uint32_t*>(&h2);
              }
              *reinterpret_cast<uint4*>(p + e) = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
        if (seen >= 0 && x == 0) {
          if (!whole) a.part_s[(long long)slot * kQrRows + t] = lse2;
          else if (a.lse_out) a.lse_out[(long long)head * a.n_rows + row] = lse2 * 0.6931471805599453f;
        }
        tc_fence_before();
      }
      asm volatile("bar.sync 2, 256;" ::: "memory");       // O and the sums have been read by both groups
      more = g.next(a, st);
    }
  } else if (warp < 16) {
    reg_dealloc<80>();
    // ================= tiles: 8 bits -> fp16 in shared memory; four warps for K, four for V =================
    constexpr int kPieces = D / 16, kAtOnce = 128 / kPieces, kTrips = kQrTile / kAtOnce;      // 16-byte pieces of a token; tokens that four warps bring at once
    static_assert(kAtOnce % 8 == 0, "rows of the same swizzle");
    const bool of_k = warp < 12;
    const int ct = tid & 127, cw = warp & 3;
    // A piece becomes two chunks of 16 bytes.  Eight lanes: two tokens of four pieces (64 dims), whose chunks lie in eight different groups of banks.
    const int my_token = D == 128 ? (ct >> 4) * 2 + ((ct >> 2) & 1) : ct >> 2, half = D == 128 ? (ct >> 3) & 1 : 0, my_piece = (ct & 3) + 4 * half;
    const uint32_t place0 = (uint32_t)(((ct & 3) * 2) ^ (my_token & 7)) << 4;
    const uint32_t full = of_k ? full_k : full_v, empty = of_k ? empty_k : empty_v;
    const uint32_t raw_at = L::kRaw + (of_k ? 0 : L::kRawTile) + ct * 16;       // this thread's pieces, kTrips of a tile, 128 x 16 bytes apart; two tiles
    uint8_t* to_tile = base_ptr + (of_k ? 0 : L::kV) + half * L::kHalfBytes + my_token * 128;
    bool ok = true;
    uint32_t jj = 0;
    for (bool more = true; more && ok; more = ok && g.next(a, st)) {
      const int* pages = a.table + g.seq * a.table_stride;
      const uint8_t* from = (of_k ? a.k : a.v) + g.hd * (long long)a.head_stride;
      const long long lane_off = my_token % 16 * a.token_stride + my_piece * 16;
      auto block_number = [&](int j) -> int {            // of 16 tokens of tile j, for lanes 0 to 7; -1: behind the end
        const long long t = (long long)j * kQrTile + lane * 16;
        return lane < 8 && j < g.j1 && t < g.s.len ? pages[t >> a.block_shift] : -1;
      };
      auto issue = [&](int j, int id) {                  // id: of this lane's 16 tokens
        const uint32_t dst = base + raw_at + ((jj + j - g.j0) & 1) * (L::kRawTile / 2);
        if (j < g.j1) {
          const int left = (int)min((long long)kQrTile, g.s.len - (long long)j * kQrTile);
          const bool known = (unsigned)id < (unsigned)a.n_blocks;
          const unsigned long long mine = known ? reinterpret_cast<unsigned long long>(from + id * a.block_stride + ((j * kQrTile + (lane & 7) * 16) & bs_mask) * a.token_stride) : 0ull;
#pragma unroll 8
          for (int i = 0; i < kTrips; ++i) {
            const int token = i * kAtOnce + my_token;
            const unsigned long long p = __shfl_sync(0xffffffffu, mine, token >> 4);
            const bool there = token < left && p != 0;
            copy_16(dst + i * 2048, there ? reinterpret_cast<const uint8_t*>(p) + lane_off : a.k, there ? 16 : 0);
          }
        }
        copies_commit();
      };
      auto exponents = [&](int j, int ids, int* ek, int* ev) -> bool {       // of token ct; false: none
        const int id = __shfl_sync(0xffffffffu, ids, ct >> 4);
        const long long t = (long long)j * kQrTile + ct;
        const bool inside = j < g.j1 && t < g.s.len, there = inside && (unsigned)id < (unsigned)a.n_blocks;
        if (inside && !there && (ct & 15) == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ATTN, id, a.n_blocks);
        *ek = 0; *ev = -200;
        if (there) {
          const long long at = (((long long)id * a.Hkv + g.hd) << a.block_shift) + ((int)t & bs_mask);
          *ek = a.k_exp[at];
          *ev = a.v_exp[at];
        }
        return there;
      };
      const int n = g.j1 - g.j0;
      int e_run = -200, ek = 0, ev = 0, id1 = block_number(g.j0), id2 = block_number(g.j0 + 1);
      issue(g.j0, id1);
      issue(g.j0 + 1, id2);
      bool there = of_k ? exponents(g.j0, id1, &ek, &ev) : false;
      id1 = id2;                                         // of tile i + 1
      id2 = block_number(g.j0 + 2);                      // of tile i + 2
      for (int i = 0; i < n; ++i) {
        const uint32_t u = jj + i, x = u & 1;
        const int ring = u & 3, id3 = block_number(g.j0 + i + 3);
        copies_wait<1>();                                // (of this thread's own pieces)
        if (u > 1) {
          ok = __all_sync(0xffffffffu, mbar_wait(empty + 8 * x, ((u >> 1) & 1) ^ 1u, abort_flag));
          if (!ok && !of_k) break;
        }
        uint8_t* to = to_tile + x * L::kTileBytes;
        const uint8_t* raw = base_ptr + raw_at + x * (L::kRawTile / 2);
#pragma unroll 8
        for (int c = 0; c < (ok ? kTrips : 0); ++c) {    // (kAtOnce tokens on, a row's chunks lie in the same order)
          uint4 h[2];
          to_half_16<TYPE>(*reinterpret_cast<const uint4*>(raw + c * 2048), h);
          *reinterpret_cast<uint4*>(to + c * kAtOnce * 128 + place0) = h[0];
          *reinterpret_cast<uint4*>(to + c * kAtOnce * 128 + (place0 ^ 16)) = h[1];
        }
        fence_proxy_async_smem();
        mbar_arrive(full + 8 * x);
        issue(g.j0 + i + 2, id2);
        if (of_k) {
          const int ev_max = __reduce_max_sync(0xffffffffu, ev == kExpNone ? -200 : ev);
          const int ek_max = __reduce_max_sync(0xffffffffu, ek);
          if (lane == 0) { largest_s[x][cw] = ev_max; largest_k_s[x][cw] = ek_max; }      // (two: a warp may be a tile ahead)
          ok = meet<1, 128>(ok);
          if (!ok) break;
          e_run = max(max(e_run, max(largest_s[x][0], largest_s[x][1])), max(largest_s[x][2], largest_s[x][3]));
          const int e_now = max(e_run, kExpLeast);       // (no token yet: anything)
          float* ks = reinterpret_cast<float*>(base_ptr + L::kScale) + ring * 3 * kQrTile;
          const float nan = __uint_as_float(0x7fc00000u);
          const int down = ev - e_now + (int)kQrShift;   // (far below: nothing)
          const int over = max(0, max(max(largest_k_s[x][0], largest_k_s[x][1]), max(largest_k_s[x][2], largest_k_s[x][3])) - kQrKeyMost);
          const float key_scale = over == 0 || ek == kExpNone ? exp_scale(ek) : ek - over > -127 ? __uint_as_float((uint32_t)(ek - over + 127) << 23) : __uint_as_float(1u << (ek - over + 149));
          ks[ct] = there ? key_scale : 0.f;
          ks[kQrTile + ct] = !there ? 0.f : ev == kExpNone ? nan : down < -126 ? 0.f : __uint_as_float((uint32_t)(down + 127) << 23);
          // (who reads the second factors sees nothing of a warp that has none to write)
          if (__any_sync(0xffffffffu, !there || ev == kExpNone || down < (int)kQrShift - kQrNear))
            ks[2 * kQrTile + ct] = !there ? 0.f : ev == kExpNone ? nan : __uint_as_float((uint32_t)(min(down + kQrBelow, 127) + 127) << 23);
          const uint32_t gone = __ballot_sync(0xffffffffu, !there), no_number = __ballot_sync(0xffffffffu, there && ev == kExpNone);
          if (lane == 0) { gone_s[ring][cw] = gone; nan_s[ring][cw] = no_number; }
          if (ct == 0) { e_s[u & 7] = e_now; over_s[ring] = over; }
          mbar_arrive(bar_scale + 8 * ring);
          there = exponents(g.j0 + i + 1, id1, &ek, &ev);
        }
        id1 = id2;
        id2 = id3;
      }
      jj += n;
      copies_wait<0>();
    }
    // the last products' arrivals come before the block goes
    for (uint32_t b = jj > 2 ? jj - 2 : 0; ok && b < jj; ++b)
      ok = mbar_wait(empty + 8 * (b & 1), (b >> 1) & 1, abort_flag);
  } else {
    reg_dealloc<48>();
    if (warp == 16) {
    // ================= products: the whole warp, one lane issues =================
    constexpr uint32_t idesc_qk = idesc_f16_f32(kQrRows, kQrTile, 0), idesc_pv = idesc_f16_f32(kQrRows, D, 1);
    constexpr uint32_t hi = desc_hi_sw128(1024);
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity & 1u, abort_flag)); };
    uint32_t jj = 0, task = 0;
    bool ok = true;
    for (bool more = true; more && ok; ++task) {
      const int n = g.j1 - g.j0;
      auto scores = [&](uint32_t u) -> bool {             // S = Q K^T of tile u
        const uint32_t x = u & 1, ph = u >> 1;
        if (!wait(full_k + 8 * x, ph)) return false;
        if (u > 1 && !wait(bar_o + 8 * x, ph - 1u)) return false;   // P of the tile that had this place has been used
        tc_fence_after();
        warp_mma_ts_kmajor<L::kHalves>(tmem_base + x * 128, tmem_base + kQ, desc_lo(base + x * L::kTileBytes, 16), hi, idesc_qk);
        warp_mma_commit(empty_k + 8 * x);
        warp_mma_commit(bar_s + 8 * x);
        return true;
      };
      ok = wait(bar_q, task);
      if (ok) ok = scores(jj);
      for (int j = 0; ok && j < n; ++j, ++jj) {
        if (j + 1 < n && !(ok = scores(jj + 1))) break;
        const uint32_t x = jj & 1, ph = jj >> 1;
        if (!(ok = wait(full_v + 8 * x, ph))) break;
        if (!(ok = wait(bar_p, jj))) break;
        tc_fence_after();
        warp_mma_ts_mnmajor(tmem_base + kO, tmem_base + x * 128, desc_lo(base + L::kV + x * L::kTileBytes, L::kHalfBytes), hi, idesc_pv, j > 0 ? 1u : 0u);
        warp_mma_commit(empty_v + 8 * x);
        warp_mma_commit(bar_o + 8 * x);
      }
      more = g.next(a, st);
    }
    }
  }
  // ---- teardown ----
  tc_fence_before();
  __syncthreads();
  if (abort_s) {
    if (tid == 0) { report(st, RELAXKV_ERR_TIMEOUT, KID_QUANTIZED_ATTN, (int)blockIdx.x, 0); a.chain[blockIdx.x].c0 = -1; }
    const uint64_t t0 = global_timer_ns();               // products still in flight: let them land
    while (global_timer_ns() - t0 < 200000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 16) { tc_fence_after(); tmem_dealloc(tmem_base, kTmemCols); }
}

// The parts of tasks that went over several blocks: a row's parts weighed by their log-sum-exps, one warp per row at a time.  The blocks c0 <= b < c1 of a task share its rows
// (of 32 warps: a row is a chain of dependent reads, and a task of two parts has one block for its 128 rows; 8 warps and a look at each row's length took 15 us more for 200
// rows over 900 tokens).
constexpr int kQrJoinWarps = 32, kQrJoinBatch = 4;
template <int D>
__global__ void __launch_bounds__(kQrJoinWarps * 32)
quantized_rows_join_kernel(const __grid_constant__ QuantAttnArgs a, DeviceStatus* st) {
  constexpr int kPer = D / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  griddep_launch();
  griddep_wait();
  const Chain ch = a.chain[blockIdx.x];
  if (ch.c0 < 0 || *reinterpret_cast<volatile int*>(&st->status) == RELAXKV_ERR_TIMEOUT) return;
  const int parts = ch.c1 - ch.c0 + 1, step = (parts - 1) * kQrJoinWarps;
  for (int col = ((int)blockIdx.x - ch.c0) * kQrJoinWarps + warp; col < ch.cols; col += step) {
    float m = kNothing, den = 0.f, acc[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = 0.f;
    const int r = col / a.G, head = ch.head * a.G + col - r * a.G;
    const long long row = ch.row + r;
    if (!(a.chain[blockIdx.x].live[col >> 5] >> (col & 31) & 1)) continue;           // (the row is left alone)
    for (int p0 = 0; p0 < parts; p0 += kQrJoinBatch) {
      float l[kQrJoinBatch], v[kQrJoinBatch][kPer];
#pragma unroll
      for (int b = 0; b < kQrJoinBatch; ++b) {
        const int p = p0 + b;
        if (p >= parts) break;
        const long long at = ((long long)(p == 0 ? 2 * ch.c0 + 1 : 2 * (ch.c0 + p))) * kQrRows + col;
        l[b] = a.part_s[at];
        if constexpr (kPer == 4) *reinterpret_cast<float4*>(v[b]) = *reinterpret_cast<const float4*>(a.part_o + at * D + lane * kPer);
        else *reinterpret_cast<float2*>(v[b]) = *reinterpret_cast<const float2*>(a.part_o + at * D + lane * kPer);
      }
#pragma unroll
      for (int b = 0; b < kQrJoinBatch; ++b) {
        if (p0 + b >= parts) break;
        if (l[b] == -INFINITY) continue;
        const float now = fmaxf(m, l[b]), was = fast_exp2(m - now), w = fast_exp2(l[b] - now), w8 = w * 0x1p-8f;      // (the sum of 148 parts at most stays within fp32)
        den = den * was + w;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] = acc[e] * was + v[b][e] * w8;
        m = now;
      }
    }
    const bool none = den == 0.f;
    const float inv = none ? 0.f : one_over(den);
    uint32_t packed[kPer / 2];
#pragma unroll
    for (int e = 0; e < kPer; e += 2) {
      const __nv_bfloat162 h2 = __floats2bfloat162_rn(acc[e] * inv * 0x1p8f, acc[e + 1] * inv * 0x1p8f);
      packed[e / 2] = *reinterpret_cast<const uint32_t*>(&h2);
    }
    uint16_t* o = a.out + (row * a.H + head) * D + lane * kPer;
    if constexpr (kPer == 4) *reinterpret_cast<uint2*>(o) = make_uint2(packed[0], packed[1]);
    else *reinterpret_cast<uint32_t*>(o) = packed[0];
    if (lane == 0 && a.lse_out) a.lse_out[(long long)head * a.n_rows + row] = none ? -INFINITY : (m + log2_of(den)) * 0.6931471805599453f;
  }
}

template <int D, int TYPE>
static cudaError_t launch_rows(const QuantAttnArgs& a, int sms, DeviceStatus* st, cudaStream_t stream) {
  static std::atomic<int> attr_done[kMaxDevices];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || dev < 0 || dev >= kMaxDevices) return e != cudaSuccess ? e : cudaErrorInvalidDevice;
  auto kern = quantized_rows_kernel<D, TYPE>;
  if (!attr_done[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, QrSmem<D>::kDynamic);
    if (e != cudaSuccess) return e;
    attr_done[dev].store(1, std::memory_order_release);
  }
  const int blocks = std::min(sms, kQrBlocks);
  e = launch_chained(kern, dim3((unsigned)blocks), kQrThreads, QrSmem<D>::kDynamic, stream, a, st);
  if (e != cudaSuccess) return e;
  auto join = quantized_rows_join_kernel<D>;
  return launch_chained(join, dim3((unsigned)blocks), kQrJoinWarps * 32, 0, stream, a, st);
}

cudaError_t launch_quantized_rows(const QuantAttnArgs& a, int head_dim, int type, int sms, DeviceStatus* st, cudaStream_t stream) {
  if (head_dim == 128) return type == RELAXKV_INT8 ? launch_rows<128, RELAXKV_INT8>(a, sms, st, stream) : launch_rows<128, RELAXKV_E4M3>(a, sms, st, stream);
  return type == RELAXKV_INT8 ? launch_rows<64, RELAXKV_INT8>(a, sms, st, stream) : launch_rows<64, RELAXKV_E4M3>(a, sms, st, stream);
}

}  // namespace relaxkv
