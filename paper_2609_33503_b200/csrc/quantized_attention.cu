// Attention of a step's rows over their sequence's tokens in the 8-bit store (relaxkv_quantized_attention).
//
// Every key and value meets the few rows and heads that read its KV head once: bound by the bytes of K and V.  Tokens are the 16
// rows of the warp-level MMA and (row, head) pairs its 8 columns, S^T = K Q^T and O^T += V^T P^T: a group of 4 or 5 heads fills
// half of it (as the 16 rows of the usual order a quarter), and what is made of a byte of K or V is used for NT column tiles.
// Bytes become fp16 in registers, exactly: two instructions for two of them (the byte under the exponent of 1024, minus that; or
// the hardware's conversion of e4m3).  Q becomes fp16 exactly, too, scaled by a power of two per head; scores get the exponent of
// their token's keys behind the product.  The exponents of the values are weighed with the scores: p'_t = 2^(s_t + e_t - max of
// that + 14), so that weights stay within fp16 whatever the exponents are, and are rounded to 11 bits; the sum of the weights is
// kept beside it in fp32, with a maximum of its own.  P^T comes out of the first product as rows of tokens and goes into the second
// as columns of them: one 8 x 8 transposition per 8 tokens.
//
// A warp streams 32 tokens at a time through a ring of its own in shared memory (16-byte asynchronous copies, no barrier between
// warps; what lies behind a sequence's end is filled with zeros and never read): twelve warps to an SM with two tiles of 8 KB in
// flight each, eight with three where a block has more than eight columns. The work of a call - (sequence, KV head, row tile, 32
// tokens), in this order - is cut into equal shares, one per block, found on the device from the lengths; a task counts eight units
// more, the time of its start and end.  A block's first and last task may be parts of one, whose results a second small kernel
// joins in the order of the blocks.  The next task's first copies are on their way while a task's results are added up.  Calls of
// few short sequences give a cluster of up to eight blocks to each row tile and KV head, which joins within itself: one launch.
// More than 32 columns to a sequence go to the kernel of many rows (quantized_rows_sm100.cu).
//
// Measured (D 128, calls among others on changing inputs): one sequence of 128 K of 32 / 8 heads 60 to 63 us
// (4.3 to 4.5 TB/s), 64 of up to 4 K of 40 / 8 heads, tokens of a head side by side, 62 (4.7 TB/s), 16 of up to 8 K 40, three rows
// of eight sequences of 8 K to 64 K 112 to 118 (4.4 to 4.6 TB/s), 1 K of 4 / 1 heads 6.5. Blocks ask for their first copies 3.8 us
// after they may begin (arguments, lengths and block numbers, one read behind the other), half of them have done their last tile 10
// us before the last one has (64 of up to 4 K: 8; they began alike, but had fewer of the late copies), the last results take 1.5 us
// more and the join 4 to 5.
#include "quantized_attention.cuh"

namespace relaxkv {

constexpr int kQaWarps = 4, kQaThreads = kQaWarps * 32, kQaTile = 32;
constexpr int kQaBlocks = 3 * 148;               // blocks that a call is cut into, at most (a workspace size does not depend on the device asked)
constexpr int kQaColsMost = 32;                  // (row, head) columns of a block, at most
constexpr float kPShift = 14.f;                  // the largest weight is 2^14

template <int D, int NT>
struct QaSmem {
  static constexpr int kBlocksPerSm = NT == 1 ? 3 : 2, kStages = NT == 1 ? 2 : 3;
  static constexpr int kTile = kQaTile * D;                          // bytes of a tile of keys
  static constexpr int kV = kTile, kExp = 2 * kTile;                 // K | V | exponents of K, of V
  static constexpr int kStage = kExp + 128;
  static constexpr int kWarp = kStages * kStage;
  static constexpr int kTotal = kQaWarps * kWarp;
  // Where the warps exchange their results: the last stages of every ring, while the first kBefore are filled for the next task.
  static constexpr int kResult = (D / 16 - D / 16 / kQaWarps) * NT * 512;
  static constexpr int kBefore = kStages - (kResult + kStage - 1) / kStage;
  static_assert(kBefore >= 1, "a warp's results leave a stage");
};

// Place of 16-byte piece c of token t of a tile.  The eight rows of a matrix are tokens 4 r + j, so that a lane's four tokens are neighbours (their exponents are one
// word); the same piece of them lies in eight different groups of banks.
template <int D>
__device__ __forceinline__ int swizzled(int t, int c) {
  return D == 128 ? t * 128 + ((c ^ ((t >> 2) & 7)) << 4) : ((t & ~1) | ((t ^ (t >> 4)) & 1)) * 64 + ((c ^ ((t >> 2) & 3)) << 4);
}

__device__ __forceinline__ void load_matrices(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_matrices_trans(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t r) {
  uint32_t t;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(r));
  return t;
}
__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Bytes 0, 1 and 2, 3 of w as fp16 pairs (keys), bytes 0, 2 and 1, 3 (values, after the transposition of pairs of dims).
template <int TYPE>
__device__ __forceinline__ void key_pairs(uint32_t w, uint32_t* lo, uint32_t* hi) {
  if constexpr (TYPE == RELAXKV_INT8) {
    w ^= 0x80808080u;
    *lo = int8_to_half2<0x4140>(w); *hi = int8_to_half2<0x4342>(w);
  } else { *lo = e4m3_to_half2(w, 0); *hi = e4m3_to_half2(w, 1); }
}
template <int TYPE>
__device__ __forceinline__ void value_pairs(uint32_t w, uint32_t* even, uint32_t* odd) {
  if constexpr (TYPE == RELAXKV_INT8) {
    w ^= 0x80808080u;
    *even = int8_to_half2<0x4240>(w); *odd = int8_to_half2<0x4341>(w);
  } else {
    w = __byte_perm(w, 0, 0x3120);
    *even = e4m3_to_half2(w, 0); *odd = e4m3_to_half2(w, 1);
  }
}

__device__ __forceinline__ float max_over_tokens(float x) {              // lanes of one column
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
using QaWalk = Walk<kQaTile, 8, 8, kQaThreads>;

// What is known of a column: a maximum of the scores, the reference of scores + exponents of the values (in log2 units), sum of the weights.
struct ColStats { float m, mp, z; };

__device__ __forceinline__ bool some_byte_below_2(uint32_t w) {
  const uint32_t x = w & 0xfefefefeu;
  return ((x - 0x01010101u) & ~x & 0x80808080u) != 0;
}

template <int D, int TYPE, int NT, bool WHOLE>
__global__ void __launch_bounds__(kQaThreads, QaSmem<D, NT>::kBlocksPerSm)
quantized_attention_kernel(const __grid_constant__ QuantAttnArgs a, DeviceStatus* st) {
  using L = QaSmem<D, NT>;
  constexpr int kStages = L::kStages;
  constexpr int kCols = 8 * NT, kChunks = D / 16;                     // columns of the block; 16-dim pieces of a head
  constexpr bool kQInRegs = NT <= 2;
  constexpr int kOwn = kChunks / kQaWarps;                            // pieces of the result that a warp adds up
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ ColStats stats_s[kQaWarps][kCols], result_s[WHOLE ? kCols : 1];
  static_assert(kOwn * NT * 512 <= L::kBefore * L::kStage, "a warp's pieces of a cluster's part");
  __shared__ int len_s[kCols];                                        // tokens that a column sees; -1: none, and it is not written
  __shared__ float qscale_s[kCols];
  __shared__ int at_s[kCols];                                         // its row * H + head (less than 2^31: see the host's limit); -1: not written
  __shared__ __align__(16) uint2 q_s[kQInRegs ? 1 : kChunks][kQInRegs ? 1 : NT][32];
  __shared__ QaWalk::Shared walk_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gid = lane >> 2, tig = lane & 3;
  const uint32_t ring = ptx::smem_u32(smem) + warp * L::kWarp;
  uint8_t* ring_ptr = smem + warp * L::kWarp;
  const int G = a.G, rpt = a.rows_per_tile, bs_mask = (1 << a.block_shift) - 1;
  if (!WHOLE) griddep_launch();                                       // (the join's blocks come as these leave, and wait)
  griddep_wait();

  // ---- this block's share ----
  QaWalk g;
  int rank = 0;                                                       // of this block in its cluster
  // WHOLE: a block, or a cluster, per rows_at_once rows and KV head; the first of a row tile's rows takes them all.
  long long row = 0, row_end = 0;
  auto find = [&]() -> bool {                                         // the next such row
    for (bool once = true; NT > 1 ? row < row_end : once; ++row, once = false) {      // (NT 1: one row)
      // (of as many sequences as rows, each row is mostly the only one of its sequence: what is known then comes with its number, not behind it; 64 x 300 tokens 18.8 us in
      // place of 20.5.  The same for any number of rows, all alike, gained nothing: 19.6, and 25.9 of 25.6 for six rows of 43 short sequences.)
      const bool one_each = a.n_rows == a.n_seq;
      int first1 = 0, end1 = 0, len1 = 0;
      if (one_each) { first1 = a.row_cu[row]; end1 = a.row_cu[row + 1]; len1 = a.row_len[row]; }
      g.seq = a.row_seq[row];
      const bool tell = tid == 0 && g.hd == 0 && rank == 0;
      if (row >= a.row_cu[a.n_seq] || g.seq == -1) continue;
      if (g.seq < 0 || g.seq >= a.n_seq) {
        if (tell) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ATTN, g.seq, (int)row);
        continue;
      }
      g.s = one_each && g.seq == row && first1 == row && end1 == row + 1 ? rows_with(a, g.seq, first1, end1, len1, tell, st) : rows_of(a, g.seq, -1, 0, tell, st);
      if (g.s.n == 0) continue;
      if (row < g.s.first || row >= g.s.first + g.s.n) {
        if (tell) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ATTN, g.seq, (int)row);
        continue;
      }
      g.tile = (int)(row - g.s.first) / rpt;
      const long long first = g.s.first + (long long)g.tile * rpt;
      bool another = false;
      for (long long r = first; r < row && !another; ++r) another = a.row_seq[r] == g.seq;
      if (another) continue;
      g.tiles = QaWalk::tiles_of(g.s.len);
      const int each = (g.tiles + a.split - 1) / a.split;
      g.j0 = min(g.tiles, rank * each);
      g.j1 = min(g.tiles, g.j0 + each);
      row = min(first + rpt, (long long)g.s.first + g.s.n);           // (what is between is of this tile, or reported with it)
      return true;
    }
    return false;
  };
  if constexpr (WHOLE) {
    const int unit = (int)blockIdx.x / a.split;
    const long long rows = unit / a.Hkv;
    rank = (int)blockIdx.x - unit * a.split;
    g.hd = unit - (int)rows * a.Hkv;
    row = rows * a.rows_at_once;
    row_end = min(row + a.rows_at_once, a.n_rows);
    if (!find()) return;                                              // (with it the other blocks of its cluster)
  } else {
    if (!g.begin(a, walk_s, st)) {                                    // (or it ends before the first tile of its only task)
      if (tid == 0) a.chain[blockIdx.x].c0 = -1;
      return;
    }
  }

  // ---- copies: lane l has piece l % (D / 16) of every (512 / D)-th token; block numbers of sixteen tiles at a time, one lane each half ----
  constexpr int kPieces = D / 16, kTokensAtOnce = 32 / kPieces, kCopies = 16 / kTokensAtOnce;
  const int my_token = lane / kPieces, my_piece = lane % kPieces;
  const long long v_off = a.v - a.k, step = kTokensAtOnce * a.token_stride;
  const uint8_t* k_all = a.k + my_token * a.token_stride + my_piece * 16;
  auto tiles_mine = [&]() { return g.j1 - g.j0 > warp ? (g.j1 - g.j0 - warp + kQaWarps - 1) / kQaWarps : 0; };      // tiles j0 + warp, + 4, ..
  int n_mine = tiles_mine(), page = 0;

  // What has been weighed of the task's tokens.  m and z are this lane's own, of its tokens; mp is the column's: all weights of the column that meet values are 2^(s + e - mp + 14)
  float qs[NT][2], m[NT][2], mp[NT][2], z[NT][2], o[kChunks][NT][4];
  uint2 qf[kQInRegs ? kChunks : 1][kQInRegs ? NT : 1];                // the columns of Q as fragments
  int seen[NT][2], seen_all = 0;
  bool huge = false;
  // The task before, whose results are still to be added up.
  bool pending = false, pending_whole = false, more = true;
  int pending_slot = 0;
  Chain left = {-1};

  // One trip per tile: its products, then the copies of the tile that takes its place in the ring.  A task's first trips have copies only; between them the results of the task
  // before are added up and the rows of this one fetched.  (Every part of the code stands here once: the instructions of a short call come from far.)
  for (int it = -kStages, stage = 0;; ++it) {
    if (it >= 0) {
      copies_wait<kStages - 1>();
      __syncwarp();
      const uint32_t kt = ring + stage * L::kStage, vt = kt + L::kV;
      const uint8_t* exps = ring_ptr + stage * L::kStage + L::kExp;
      const int t0 = (g.j0 + warp + it * kQaWarps) * kQaTile;
      const uint32_t ke = *reinterpret_cast<const uint32_t*>(exps + gid * 4) ^ 0x80808080u, ve = *reinterpret_cast<const uint32_t*>(exps + 32 + gid * 4) ^ 0x80808080u;
      // ---- S^T = K Q^T: 16 tokens by the columns, twice ----
      float sc[2][NT][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[h][nt][0] = sc[h][nt][1] = sc[h][nt][2] = sc[h][nt][3] = 0.f;
#pragma unroll
        for (int c4 = 0; c4 < kChunks / 4; ++c4) {
          uint32_t lo[4], hi[4];                                      // tokens 4 r + 2 h, 4 r + 2 h + 1
          const int t = (lane & 7) * 4 + 2 * h, c = c4 * 4 + (lane >> 3);
          load_matrices(lo, kt + swizzled<D>(t, c));
          load_matrices(hi, kt + swizzled<D>(t + 1, c));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t frag[4];
            key_pairs<TYPE>(lo[i], &frag[0], &frag[2]);
            key_pairs<TYPE>(hi[i], &frag[1], &frag[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              uint2 b;
              if constexpr (kQInRegs) b = qf[c4 * 4 + i][nt]; else b = q_s[c4 * 4 + i][nt][lane];
              mma_f16(sc[h][nt], frag, b.x, b.y);
            }
          }
        }
      }
      // ---- scores of this lane: tokens 4 gid + i, i = 2 h + y, columns 2 tig (+ 1); w: with the exponents of the values ----
      // (queries so large that a score would leave fp32 before its key's scale brings it back take 2^-64 of it first)
      if (huge) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int y = 0; y < 4; ++y) sc[h][nt][y] *= 0x1p-64f;
      }
      float vexp[4], w[NT][2][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ks = __uint_as_float((__byte_perm(ke, 0, 0x0444 | i << 12) >> 1) - 0x800000u);      // 2^e (of a key that is none, or no number: replaced below)
        vexp[i] = __uint_as_float(__byte_perm(ve, 0x4b000000u, 0x7550 | i)) - 8388736.f;     // 2^23 + byte, less 2^23 + 128
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float& v = sc[i >> 1][nt][2 * (i & 1) + x];
            v = v * qs[nt][x] * ks;
            if (huge) v *= 0x1p64f;
            w[nt][x][i] = v + vexp[i];
          }
      }
      if (__any_sync(0xffffffffu, t0 + kQaTile > seen_all || some_byte_below_2(ke) || some_byte_below_2(ve))) {      // tokens that are not seen, NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = gid * 4 + i, ek = (ke >> (8 * i)) & 255u, ev = (ve >> (8 * i)) & 255u;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float& v = sc[i >> 1][nt][2 * (i & 1) + x];
              if (ek == kExpNone + 128) v = w[nt][x][i] = __uint_as_float(0x7fc00000u);
              if (ev == kExpNone + 128) w[nt][x][i] = __uint_as_float(0x7fc00000u);
              if (ek == kNoKey + 128 || t0 + at >= seen[nt][x]) v = w[nt][x][i] = -INFINITY;
            }
        }
      }
      uint32_t pb[2][NT][2];                                          // P^T as fragments: tokens 4 r + 2 h, 4 r + 2 h + 1
      bool grown = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float ms = ptx::fmax3(ptx::fmax3(sc[0][nt][x], sc[0][nt][2 + x], sc[1][nt][x]), sc[1][nt][2 + x], m[nt][x]);
          float zz = z[nt][x] * ptx::fast_exp2(m[nt][x] - ms);
#pragma unroll
          for (int i = 0; i < 4; ++i) zz += ptx::fast_exp2(sc[i >> 1][nt][2 * (i & 1) + x] - ms);
          z[nt][x] = zz;
          m[nt][x] = ms;
          grown |= ptx::fmax3(w[nt][x][0], w[nt][x][1], fmaxf(w[nt][x][2], w[nt][x][3])) > mp[nt][x] + 1.f;       // (weights up to 2^15 are fine)
        }
      if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float mt = ptx::fmax3(w[nt][x][0], w[nt][x][1], fmaxf(w[nt][x][2], w[nt][x][3]));
            const float top = max_over_tokens(mt), now = top > mp[nt][x] + 1.f ? top : mp[nt][x];      // (what its neighbours do is nothing to a column)
            const float alpha = ptx::fast_exp2(mp[nt][x] - now);
            mp[nt][x] = now;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) { o[c][nt][x] *= alpha; o[c][nt][2 + x] *= alpha; }
          }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float ref0 = mp[nt][0] - kPShift, ref1 = mp[nt][1] - kPShift;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __half2 p = __floats2half2_rn(ptx::fast_exp2(w[nt][0][i] - ref0), ptx::fast_exp2(w[nt][1][i] - ref1));
          pb[i >> 1][nt][i & 1] = transposed(*reinterpret_cast<const uint32_t*>(&p));
        }
      }
      // ---- O^T += V^T P^T: rows of the fragment are dims 2 gid, then 2 gid + 1 of a 16-dim piece ----
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c2 = 0; c2 < kChunks / 2; ++c2) {
          uint32_t w[4];                                              // (tokens 4 r + 2 h, 4 r + 2 h + 1) of two pieces
          load_matrices_trans(w, vt + swizzled<D>((lane & 7) * 4 + 2 * h + ((lane >> 3) & 1), c2 * 2 + (lane >> 4)));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t frag[4];
            value_pairs<TYPE>(w[2 * i], &frag[0], &frag[1]);
            value_pairs<TYPE>(w[2 * i + 1], &frag[2], &frag[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_f16(o[c2 * 2 + i][nt], frag, pb[h][nt][0], pb[h][nt][1]);
          }
        }
      __syncwarp();                                                   // everyone is through with the stage
    } else if (it == L::kBefore - kStages) {
      if (pending) {
        // ---- the warps' results of the task before, added up in their order: every warp adds up a quarter of the pieces, the others' come through the rings ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float all = max_over_tokens(m[nt][x]);
            float zz = z[nt][x] * ptx::fast_exp2(m[nt][x] - all);
            zz += __shfl_xor_sync(0xffffffffu, zz, 4);
            zz += __shfl_xor_sync(0xffffffffu, zz, 8);
            zz += __shfl_xor_sync(0xffffffffu, zz, 16);
            if (gid == 0) stats_s[warp][nt * 8 + tig * 2 + x] = {all, mp[nt][x], zz};
          }
        auto place = [&](int w, int c, int nt) -> float4& {           // warp w's result of piece c, which is another's
          return reinterpret_cast<float4*>(smem + w * L::kWarp + L::kBefore * L::kStage)[((c - (c >= (w + 1) * kOwn ? kOwn : 0)) * NT + nt) * 32 + lane];
        };
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            if (c / kOwn != warp) place(warp, c, nt) = make_float4(o[c][nt][0], o[c][nt][1], o[c][nt][2], o[c][nt][3]);
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float big[2], bigp[2], zs[2], wgt[kQaWarps][2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int col = nt * 8 + tig * 2 + x;
            big[x] = bigp[x] = kNothing;
#pragma unroll
            for (int w = 0; w < kQaWarps; ++w) { big[x] = fmaxf(big[x], stats_s[w][col].m); bigp[x] = fmaxf(bigp[x], stats_s[w][col].mp); }
            zs[x] = 0.f;
#pragma unroll
            for (int w = 0; w < kQaWarps; ++w) {
              zs[x] = fmaf(stats_s[w][col].z, ptx::fast_exp2(stats_s[w][col].m - big[x]), zs[x]);
              wgt[w][x] = ptx::fast_exp2(stats_s[w][col].mp - bigp[x]);
            }
            if (!pending_whole && warp == 0 && gid == 0) {
              if constexpr (WHOLE) result_s[col] = {big[x], bigp[x], zs[x]};
              else {
                float* p = a.part_s + ((long long)pending_slot * kQaColsMost + col) * 3;
                p[0] = big[x]; p[1] = bigp[x]; p[2] = zs[x];
              }
            }
          }
          float acc[kOwn][4];
#pragma unroll
          for (int i = 0; i < kOwn; ++i) {
            acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
            for (int w = 0; w < kQaWarps; ++w) {
              float4 v;
              if (w != warp) v = place(w, warp * kOwn + i, nt);
              else {
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
                  if (c == warp * kOwn + i) v = make_float4(o[c][nt][0], o[c][nt][1], o[c][nt][2], o[c][nt][3]);
              }
              acc[i][0] = fmaf(v.x, wgt[w][0], acc[i][0]); acc[i][1] = fmaf(v.y, wgt[w][1], acc[i][1]);
              acc[i][2] = fmaf(v.z, wgt[w][0], acc[i][2]); acc[i][3] = fmaf(v.w, wgt[w][1], acc[i][3]);
            }
          }
          if (!pending_whole) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
              *(WHOLE ? reinterpret_cast<float4*>(ring_ptr) + (i * NT + nt) * 32 + lane       // (in front of the exchange)
                      : reinterpret_cast<float4*>(a.part_o + (((long long)pending_slot * kChunks + warp * kOwn + i) * NT + nt) * 128 + lane * 4)) =
                  make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
          } else {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int at = at_s[nt * 8 + tig * 2 + x];
              if (at < 0) continue;
              const bool none = zs[x] == 0.f;                         // no token at all, or none above -inf (NaN stays NaN)
              const float norm = none ? 0.f : one_over(zs[x] * 16384.f), grow = none ? 0.f : ptx::fast_exp2(bigp[x] - big[x]);
#pragma unroll
              for (int i = 0; i < kOwn; ++i)
                *reinterpret_cast<__nv_bfloat162*>(a.out + (long long)at * D + (warp * kOwn + i) * 16 + gid * 2) =
                    __floats2bfloat162_rn(acc[i][x] * norm * grow, acc[i][2 + x] * norm * grow);
              if (warp == 0 && gid == 0 && a.lse_out) {
                const int row = at / a.H;
                a.lse_out[(at - row * a.H) * a.n_rows + row] = none ? -INFINITY : (big[x] + log2_of(zs[x])) * 0.6931471805599453f;
              }
            }
          }
        }
        if (!more) break;
        __syncthreads();                                              // all of that has been read
      }
      // ---- the rows of this task: 16-dim piece c of a column, dims 4 tig .. 4 tig + 3 of it, as fp16 times 2^-exponent ----
      const long long row_first = g.s.first + (long long)g.tile * rpt;
      const int cols = min(rpt, g.s.n - g.tile * rpt) * G;
      if (tid < kCols) {
        const int r = tid / G, len = tid < cols ? row_tokens(a, g.seq, g.s, row_first + r, tid - r * G == 0 && g.hd == 0 && g.j0 == 0 && rank == 0, st) : -1;
        len_s[tid] = len;
        at_s[tid] = len < 0 ? -1 : (int)(row_first + r) * a.H + g.hd * G + tid - r * G;
      }
      if (kQInRegs || warp == 0) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int col = nt * 8 + gid, r = col / G;
          const uint16_t* q = a.q + ((row_first + r) * a.H + g.hd * G + col - r * G) * D + tig * 4;
          uint2 raw[kChunks];
          uint32_t top = 0;
#pragma unroll
          for (int c = 0; c < kChunks; ++c) raw[c] = col < cols ? *reinterpret_cast<const uint2*>(q + c * 16) : make_uint2(0u, 0u);
#pragma unroll
          for (int c = 0; c < kChunks; ++c) top = __vmaxu2(top, __vmaxu2(raw[c].x & 0x7fff7fffu, raw[c].y & 0x7fff7fffu));
          top = max(top & 0xffffu, top >> 16);
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const bool finite = top < 0x7f80u;
          const int e = max((int)(top >> 7) - 127 - 14, -120);        // the largest element comes to lie in [2^14, 2^15)
          const float inv = __uint_as_float((uint32_t)(127 - (finite ? e : 0)) << 23);
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            const __half2 x = __floats2half2_rn(__uint_as_float(raw[c].x << 16) * inv, __uint_as_float(raw[c].x & 0xffff0000u) * inv);
            const __half2 y = __floats2half2_rn(__uint_as_float(raw[c].y << 16) * inv, __uint_as_float(raw[c].y & 0xffff0000u) * inv);
            const uint2 h2 = finite ? make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y)) : make_uint2(0u, 0u);
            if constexpr (kQInRegs) qf[c][nt] = h2;
            else q_s[c][nt][lane] = h2;
          }
          if (warp == 0 && tig == 0) qscale_s[col] = finite ? __uint_as_float((uint32_t)(127 + e) << 23) * a.scale_log2 : __uint_as_float(0x7fc00000u);
        }
      }
      __syncthreads();
      seen_all = g.s.len;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int col = nt * 8 + tig * 2 + x;
          qs[nt][x] = qscale_s[col];
          seen[nt][x] = len_s[col];
          if (col < cols) seen_all = min(seen_all, seen[nt][x]);
          m[nt][x] = mp[nt][x] = kNothing;
          z[nt][x] = 0.f;
        }
      bool far = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) far |= fmaxf(qs[nt][0], qs[nt][1]) > 0x1p90f;
      huge = __any_sync(0xffffffffu, far);
      seen_all = min(seen_all, __shfl_xor_sync(0xffffffffu, seen_all, 1));
      seen_all = min(seen_all, __shfl_xor_sync(0xffffffffu, seen_all, 2));
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[c][nt][0] = o[c][nt][1] = o[c][nt][2] = o[c][nt][3] = 0.f;
    }

    // ---- copies of tile it + kStages ----
    const int ahead = it + kStages;
    if ((ahead & 15) == 0) {
      const int mine = ahead + (lane >> 1);
      page = -1;
      if (mine < n_mine) {                                            // (its tokens' numbers fit 32 bits: see the host's limit)
        const int t = (g.j0 + warp + mine * kQaWarps) * kQaTile + (lane & 1) * 16;
        if (t < g.s.len) page = a.table[g.seq * a.table_stride + (t >> a.block_shift)];
      }
    }
    if (ahead < n_mine) {
      const uint32_t dst = ring + stage * L::kStage;
      const int t0 = (g.j0 + warp + ahead * kQaWarps) * kQaTile;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int id = __shfl_sync(0xffffffffu, page, (ahead & 15) * 2 + h), t = t0 + h * 16;
        const bool there = t < g.s.len && (unsigned)id < (unsigned)a.n_blocks;
        const int valid = there ? min(16, g.s.len - t) : 0;
        const uint8_t* p = k_all + g.hd * a.head_stride + (there ? id * a.block_stride + (t & bs_mask) * a.token_stride : 0);
        if (t < g.s.len && !there && lane == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ATTN, id, a.n_blocks);
        // behind the end of the sequence, and where there is no such block: zeros, and nothing is read
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const bool some = my_token + i * kTokensAtOnce < valid;
          const uint32_t d = dst + swizzled<D>(my_token + h * 16 + i * kTokensAtOnce, my_piece);
          copy_16(d, p, some ? 16 : 0);                               // (a block has these sixteen tokens in any case)
          copy_16(d + L::kV, p + v_off, some ? 16 : 0);
          p += step;
        }
        if (lane < 2) {
          const uint32_t e = stage * L::kStage + L::kExp + lane * 32 + h * 16;
          if (there) copy_16(ring + e, (lane ? a.v_exp : a.k_exp) + ((((long long)id * a.Hkv + g.hd) << a.block_shift) + (t & bs_mask)), 16);
          else *reinterpret_cast<uint4*>(ring_ptr + e) = make_uint4(0x81818181u, 0x81818181u, 0x81818181u, 0x81818181u);
        }
      }
    }
    copies_commit();
    stage = stage + 1 == kStages ? 0 : stage + 1;

    // ---- the task ends: what comes behind it ----
    if (it >= -1 && it >= n_mine - 1) {
      copies_wait<0>();
      __syncwarp();
      pending = true;
      pending_whole = WHOLE ? a.split == 1 : g.whole();
      pending_slot = g.slot();
      more = false;
      if constexpr (!WHOLE) {
        left.row = g.s.first + g.tile * rpt;
        left.head = g.hd;
        left.cols = min(rpt, g.s.n - g.tile * rpt) * G;
        left.live[0] = __ballot_sync(0xffffffffu, lane < kCols && len_s[lane < kCols ? lane : 0] >= 0);
        left.c0 = -1;
        if (g.j1 < g.tiles) g.blocks_of(&left.c0, &left.c1);
        more = g.next(a, st);
      } else if constexpr (NT > 1) {
        if (a.split == 1) more = find();
      }
      n_mine = more ? tiles_mine() : 0;
      stage = 0;
      it = -kStages - 1;
    }
  }
  if constexpr (WHOLE) {
    if (a.split > 1) {
      // ---- the parts of the cluster's blocks, added up in their order: unit u = (16 dims, 8 columns), the warps of all blocks take them in turn ----
      ptx::cluster_sync();
      for (int u = rank * kQaWarps + warp; u < kChunks * NT; u += a.split * kQaWarps) {
        const int nt = u % NT, c = u / NT, owner = c / kOwn;
        const uint32_t from = ptx::smem_u32(smem) + owner * L::kWarp + (((c - owner * kOwn) * NT + nt) * 32 + lane) * 16;
        const uint32_t stats = ptx::smem_u32(&result_s[nt * 8 + tig * 2]);
        float sm[2] = {kNothing, kNothing}, smp[2] = {kNothing, kNothing}, sz[2] = {0.f, 0.f}, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int b = 0; b < a.split; ++b) {
          const uint32_t there = ptx::mapa_shared(from, b), of = ptx::mapa_shared(stats, b);
          const float4 v = ptx::ld_cluster_f32x4(there);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float m1 = ptx::ld_cluster_f32(of + 12 * x), mp1 = ptx::ld_cluster_f32(of + 12 * x + 4), z1 = ptx::ld_cluster_f32(of + 12 * x + 8);
            const float big = fmaxf(sm[x], m1), bigp = fmaxf(smp[x], mp1), was = ptx::fast_exp2(smp[x] - bigp), w1 = ptx::fast_exp2(mp1 - bigp);
            sz[x] = sz[x] * ptx::fast_exp2(sm[x] - big) + z1 * ptx::fast_exp2(m1 - big);
            acc[x] = acc[x] * was + (x ? v.y : v.x) * w1;
            acc[2 + x] = acc[2 + x] * was + (x ? v.w : v.z) * w1;
            sm[x] = big; smp[x] = bigp;
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int at = at_s[nt * 8 + tig * 2 + x];
          if (at < 0) continue;
          const bool none = sz[x] == 0.f;
          const float norm = none ? 0.f : one_over(sz[x] * 16384.f), grow = none ? 0.f : ptx::fast_exp2(smp[x] - sm[x]);
          *reinterpret_cast<__nv_bfloat162*>(a.out + (long long)at * D + c * 16 + gid * 2) = __floats2bfloat162_rn(acc[x] * norm * grow, acc[2 + x] * norm * grow);
          if (c == 0 && gid == 0 && a.lse_out) {
            const int row = at / a.H;
            a.lse_out[(at - row * a.H) * a.n_rows + row] = none ? -INFINITY : (sm[x] + log2_of(sz[x])) * 0.6931471805599453f;
          }
        }
      }
      ptx::cluster_sync();                                                 // nobody leaves while its part is read
    }
    __syncthreads();
    griddep_launch();
  } else if (tid == 0) a.chain[blockIdx.x] = left;
}

// The parts of tasks that went over several blocks, joined in their order.  The blocks c0 <= b < c1 that such a task leaves share its (16 dims, 8 columns) units; a block's
// warps share a unit's parts where there are fewer units than warps.
constexpr int kQjWarps = 8, kQjBatch = 8;
template <int D, int NT>
__global__ void __launch_bounds__(kQjWarps * 32)
quantized_join_kernel(const __grid_constant__ QuantAttnArgs a) {
  constexpr int kChunks = D / 16, kUnits = kChunks * NT;
  struct Joined { float m[2], mp[2], z[2], acc[4]; };
  __shared__ Joined join_s[kQjWarps][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3, G = a.G;
  griddep_launch();
  griddep_wait();
  const Chain ch = a.chain[blockIdx.x];
  if (ch.c0 < 0) return;
  const int parts = ch.c1 - ch.c0 + 1, blocks = parts - 1, me = (int)blockIdx.x - ch.c0, mine = (kUnits - me + blocks - 1) / blocks;      // units me, me + blocks, ..
  if (me >= kUnits) return;
  const int groups = max(1, kQjWarps / mine);                         // warps of a unit
  for (int u0 = 0; u0 < mine; u0 += kQjWarps / groups) {
    const int in = warp / groups, g = warp - in * groups, u = me + (u0 + in) * blocks;
    const bool has = in < kQjWarps / groups && u0 + in < mine;
    const int c = has ? u / NT : 0, nt = has ? u - c * NT : 0;
    Joined r = {{kNothing, kNothing}, {kNothing, kNothing}, {0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int p0 = g; has && p0 < parts; p0 += groups * kQjBatch) {
      float sv[kQjBatch][6];
      float4 v[kQjBatch];
#pragma unroll
      for (int b = 0; b < kQjBatch; ++b) {
        const int p = p0 + b * groups;
        if (p >= parts) break;
        const long long slot = p == 0 ? 2 * ch.c0 + 1 : 2 * (ch.c0 + p);
        const float* sp = a.part_s + (slot * kQaColsMost + nt * 8 + tig * 2) * 3;
#pragma unroll
        for (int e = 0; e < 6; e += 2) {
          const float2 y = *reinterpret_cast<const float2*>(sp + e);
          sv[b][e] = y.x; sv[b][e + 1] = y.y;
        }
        v[b] = *reinterpret_cast<const float4*>(a.part_o + ((slot * kChunks + c) * NT + nt) * 128 + lane * 4);
      }
#pragma unroll
      for (int b = 0; b < kQjBatch; ++b) {
        if (p0 + b * groups >= parts) break;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float m = fmaxf(r.m[x], sv[b][3 * x]), mp = fmaxf(r.mp[x], sv[b][3 * x + 1]);
          r.z[x] = fmaf(sv[b][3 * x + 2], ptx::fast_exp2(sv[b][3 * x] - m), r.z[x] * ptx::fast_exp2(r.m[x] - m));
          const float al = ptx::fast_exp2(r.mp[x] - mp), w = ptx::fast_exp2(sv[b][3 * x + 1] - mp);
          r.acc[x] = fmaf(w, x ? v[b].y : v[b].x, r.acc[x] * al);
          r.acc[2 + x] = fmaf(w, x ? v[b].w : v[b].z, r.acc[2 + x] * al);
          r.m[x] = m; r.mp[x] = mp;
        }
      }
    }
    if (groups > 1) {                                                 // (then this loop has one trip)
      join_s[warp][lane] = r;
      __syncthreads();
      if (has && g == 0) {
        for (int y = 1; y < groups; ++y) {
          const Joined& n = join_s[warp + y][lane];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float m = fmaxf(r.m[x], n.m[x]), mp = fmaxf(r.mp[x], n.mp[x]);
            const float wr = ptx::fast_exp2(r.mp[x] - mp), wn = ptx::fast_exp2(n.mp[x] - mp);
            r.z[x] = r.z[x] * ptx::fast_exp2(r.m[x] - m) + n.z[x] * ptx::fast_exp2(n.m[x] - m);
            r.acc[x] = r.acc[x] * wr + n.acc[x] * wn;
            r.acc[2 + x] = r.acc[2 + x] * wr + n.acc[2 + x] * wn;
            r.m[x] = m; r.mp[x] = mp;
          }
        }
      }
    }
    if (!has || g != 0) continue;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int col = nt * 8 + tig * 2 + x, rr = col / G, head = ch.head * G + col - rr * G;
      if (col >= ch.cols || !(ch.live[0] >> col & 1)) continue;
      const bool none = r.z[x] == 0.f;
      const float norm = none ? 0.f : one_over(r.z[x] * 16384.f), grow = none ? 0.f : ptx::fast_exp2(r.mp[x] - r.m[x]);
      const long long row = ch.row + rr;
      *reinterpret_cast<__nv_bfloat162*>(a.out + (row * a.H + head) * D + c * 16 + gid * 2) = __floats2bfloat162_rn(r.acc[x] * norm * grow, r.acc[2 + x] * norm * grow);
      if (c == 0 && gid == 0 && a.lse_out) a.lse_out[(long long)head * a.n_rows + row] = none ? -INFINITY : (r.m[x] + log2_of(r.z[x])) * 0.6931471805599453f;
    }
  }
}

struct QuantWs { size_t part_o, part_s, chain, total; };
static QuantWs quant_ws(int D) {
  QuantWs w{};
  size_t at = 0;
  const size_t cols = 2 * std::max<size_t>(kQaBlocks * kQaColsMost, kQrBlocks * kQrRows);       // two parts of a block
  w.part_o = at; at = align_up(at + cols * D * 4, 256);
  w.part_s = at; at = align_up(at + cols * 12, 256);
  w.chain = at; at = align_up(at + (size_t)kQaBlocks * sizeof(Chain), 256);
  w.total = at;
  return w;
}

template <int D, int TYPE, int NT, bool WHOLE>
static cudaError_t launch_attend(const QuantAttnArgs& a, long long blocks, DeviceStatus* st, cudaStream_t stream) {
  static std::atomic<int> attr_done[kMaxDevices];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || dev < 0 || dev >= kMaxDevices) return e != cudaSuccess ? e : cudaErrorInvalidDevice;
  auto kern = quantized_attention_kernel<D, TYPE, NT, WHOLE>;
  if (!attr_done[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (QaSmem<D, NT>::kTotal));
    if (e != cudaSuccess) return e;
    attr_done[dev].store(1, std::memory_order_release);
  }
  return launch_chained_clusters(WHOLE ? a.split : 1, kern, dim3((unsigned)blocks), kQaThreads, (QaSmem<D, NT>::kTotal), stream, a, st);
}
template <int D, int NT>
static cudaError_t launch_attend_n(int type, bool whole, const QuantAttnArgs& a, int sms, DeviceStatus* st, cudaStream_t stream) {
  const bool int8 = type == RELAXKV_INT8;
  if (!whole) {
    const int blocks = std::min(kQaBlocks, QaSmem<D, NT>::kBlocksPerSm * sms);
    const cudaError_t e = int8 ? launch_attend<D, RELAXKV_INT8, NT, false>(a, blocks, st, stream) : launch_attend<D, RELAXKV_E4M3, NT, false>(a, blocks, st, stream);
    if (e != cudaSuccess) return e;
    auto kern = quantized_join_kernel<D, NT>;
    return launch_chained(kern, dim3((unsigned)blocks), kQjWarps * 32, 0, stream, a);
  }
  const long long blocks = (a.n_rows + a.rows_at_once - 1) / a.rows_at_once * a.Hkv * a.split;
  return int8 ? launch_attend<D, RELAXKV_INT8, NT, true>(a, blocks, st, stream) : launch_attend<D, RELAXKV_E4M3, NT, true>(a, blocks, st, stream);
}
template <int D>
static cudaError_t launch_attend_d(int nt, int type, bool whole, const QuantAttnArgs& a, int sms, DeviceStatus* st, cudaStream_t stream) {
  return nt == 1   ? launch_attend_n<D, 1>(type, whole, a, sms, st, stream)
         : nt == 2 ? launch_attend_n<D, 2>(type, whole, a, sms, st, stream)
         : nt == 3 ? launch_attend_n<D, 3>(type, whole, a, sms, st, stream) : launch_attend_n<D, 4>(type, whole, a, sms, st, stream);
}

}  // namespace relaxkv

using namespace relaxkv;

extern "C" size_t relaxkv_quantized_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 16 || (head_dim != 64 && head_dim != 128)) return 0;
  return quant_ws(head_dim).total;
}

extern "C" relaxkv_status relaxkv_quantized_attention(
    const relaxkv_quantized_cache* store, const relaxkv_continuation_rows* r, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float softmax_scale,
    const void* q, void* out, float* lse_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_quantized_attention");
  if (n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || !(softmax_scale > 0.f)) return RELAXKV_ERR_INVALID_ARG;
  if (n_q_heads / n_kv_heads > 16 || (head_dim != 64 && head_dim != 128)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  const relaxkv_status rc = check_quantized(store, n_kv_heads, head_dim);
  if (rc != RELAXKV_OK) return rc;
  if (!r || !r->row_cu || !r->row_seq || !r->row_len || r->n_seq < 1 || r->n_rows < 0 || r->max_len < 0) return RELAXKV_ERR_INVALID_ARG;
  if (r->n_seq > kQaSeqsMost || r->max_len > kContTokensMost || r->n_rows > 0x7fffffffLL / (n_q_heads * 2)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (r->max_len > 0 && (!r->block_table || r->table_width < 1 || r->table_stride < r->table_width)) return RELAXKV_ERR_INVALID_ARG;
  if (!q || !out || q == out || !aligned16(q) || !aligned16(out)) return RELAXKV_ERR_INVALID_ARG;
  const QuantWs ws = quant_ws(head_dim);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return RELAXKV_ERR_INVALID_ARG;
  if (workspace_bytes < ws.total) return RELAXKV_ERR_WORKSPACE_TOO_SMALL;
  if (r->n_rows == 0) return RELAXKV_OK;
  DeviceStatus* st = status_word();
  const int sms = sm_count_of_current_device();
  if (!st || sms <= 0) return RELAXKV_ERR_CUDA;
  QuantAttnArgs a = {};
  a.q = static_cast<const uint16_t*>(q); a.out = static_cast<uint16_t*>(out); a.lse_out = lse_out;
  a.k = static_cast<const uint8_t*>(store->k); a.v = static_cast<const uint8_t*>(store->v); a.k_exp = store->k_exp; a.v_exp = store->v_exp;
  a.row_cu = r->row_cu; a.row_seq = r->row_seq; a.row_len = r->row_len; a.table = r->block_table;
  uint8_t* w = static_cast<uint8_t*>(workspace);
  a.part_o = reinterpret_cast<float*>(w + ws.part_o); a.part_s = reinterpret_cast<float*>(w + ws.part_s); a.chain = reinterpret_cast<Chain*>(w + ws.chain);
  a.block_stride = store->block_stride; a.token_stride = store->token_stride; a.head_stride = store->head_stride;
  a.table_stride = r->table_stride; a.n_rows = r->n_rows;
  a.table_width = r->table_width; a.n_seq = r->n_seq; a.n_blocks = store->n_blocks; a.block_shift = 31 - __builtin_clz((unsigned)store->block_size);
  a.max_len = r->max_len; a.H = n_q_heads; a.Hkv = n_kv_heads; a.G = n_q_heads / n_kv_heads;
  a.scale_log2 = softmax_scale * 1.4426950408889634f;
  // Column tiles by the rows of a sequence, on average: as few as hold them (four rows of 40 / 8 heads over 10 x 2000 tokens in three tiles 31.4 us, in four 36.7).
  const long long cols = (long long)a.G * ((r->n_rows + r->n_seq - 1) / r->n_seq);
  const int nt = cols <= 24 ? (int)(cols + 7) / 8 : 4;
  a.rows_per_tile = 8 * nt / a.G;
  // Blocks of a row tile and KV head: as many as leave each warp two tiles, where that many run at once.
  const long long items = r->n_rows * a.Hkv, tiles = (r->max_len + kQaTile - 1LL) / kQaTile;
  a.split = 1;
  while (a.split < 8 && 2 * a.split * items <= 2 * sms && 2 * a.split * kQaWarps <= tiles) a.split *= 2;
  // Where sequences have as many rows each, the next row tile begins as many further on: a block for each row would mostly be one that has nothing to do (six rows of 29 sequences of 12
  // tokens 12.0 us, so 18.6; three of 13 of 600 13.0, 15.3).  One column tile: little difference, and such blocks leave soon (two rows of 64 of 500 tokens 25.8, so 25.2).
  a.rows_at_once = nt > 1 && a.split == 1 ? (int)std::max(1LL, (long long)r->n_rows / r->n_seq) : 1;
  const bool whole = tiles <= (a.split > 1 ? 16LL * a.split : 32) && items * a.split <= 0x7fffffffLL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // More columns than one block holds: 128 at a time on the tensor cores, which takes less time than tokens brought several times (57 rows of 4 heads a group over 8 x 900
  // tokens 46 against 78 us, 20 over 16 x 300 19 against 40, 16 over 8 x 4 K 51 against 68, 30 over 3000 23.4 against 24.5; of up to 32 columns it takes more: 6 rows over 16 x 3000
  // tokens 69 against 49.5 us, over 8 K 24.7 against 20.7).
  if (cols > kQaColsMost) {
    a.rows_per_tile = kQrRows / a.G;
    return cuda_ok(launch_quantized_rows(a, head_dim, store->type, sms, st, s));
  }
  return cuda_ok(head_dim == 128 ? launch_attend_d<128>(nt, store->type, whole, a, sms, st, s) : launch_attend_d<64>(nt, store->type, whole, a, sms, st, s));
}
