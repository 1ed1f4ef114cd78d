// Context blocks by a cheap score: 8-bit bounds of every block's keys (relaxkv_block_bounds), and the blocks of the highest possible logit for
// each row and KV head (relaxkv_select_blocks).
//
// Bounds: one pass over K, bound by its bytes.  A warp has one (block, KV head): 16 lanes hold the 128 dims of a token as 16-byte pieces, so
// a load takes two tokens (four of 64 dims); maxima and minima stay packed bf16 pairs and are exact.  The scale is a power of two, so are the
// quotients, and the rounding is away from the block: the bounds remain bounds.
// Scores: sum_d max(q_d hi_d, q_d lo_d) = q+ . hi + q- . lo, a product over 2 D bytes on the tensor cores (m16n8k32, s8): rows are the heads of two
// rows of the step (of one with more than eight heads to a KV head), columns eight blocks.  The product's terms may come in any order as long as both
// sides agree, so a lane takes D / 2 bytes of its block in 16-byte loads and the queries are laid out to match.  Sums are whole numbers below 2^24:
// the scores, and with them the lists, do not depend on the order of anything.
// Selection: one block per (row, KV head); counts of digits find the lowest selected score, then every thread writes its own range's blocks in
// order.  Both launches: 4 rows of 40 / 8 heads, 512 blocks 10.3 us, 16 rows of 32 / 8 heads in two contexts of 2048 blocks 22.8: latencies
// (row -> query -> product -> score -> counts), not bytes.
#include "continuations.cuh"
#include <algorithm>

namespace relaxkv {

__device__ __forceinline__ uint32_t bmax2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t bmin2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Exponent of the smallest power of two s with |x| <= 127 s, for the bits of a finite bf16 |x|: 127 = 1.984375 * 2^6, and the next mantissa after
// that one is the last (0x7f), so adding one to the bits carries exactly when |x| is above it.  From -100 on; 0 for 0.
__device__ __forceinline__ int scale_exponent(uint32_t abs_bits) {
  return abs_bits == 0 ? 0 : max(-100, (int)((abs_bits + 1) >> 7) - 127 - 6);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }       // -100 <= e <= 127

constexpr int kBndThreads = 256;

// U: loads of a lane that travel together.  131 K tokens of 8 heads of 128 dims (268 MB) 46.4 us = 5.8 TB/s, 16 K (33.5 MB) 12.0; with sixteen loads
// 48.6 and 10.9, with thirty-two 85.2 and 12.9.
template <int D>
__global__ void __launch_bounds__(kBndThreads)
block_bounds_kernel(const uint16_t* k, long long token_stride, long long head_stride, const __grid_constant__ ContTable ct, int block_size, int Hkv,
                    int8_t* bounds, float* scale, int heads_outer) {
  constexpr int kLanes = D / 8, kTok = 32 / kLanes, U = 8;
  const int lane = threadIdx.x & 31, gl = lane % kLanes, sub = lane / kLanes;
  const long long w = (long long)blockIdx.x * (kBndThreads / 32) + (threadIdx.x >> 5);
  const int n_blocks = ct.blk_cu[ct.n_req];
  griddep_launch();
  griddep_wait();
  if (w >= (long long)n_blocks * Hkv) return;
  // warps side by side read what lies side by side in memory
  const int x = heads_outer ? (int)(w % n_blocks) : (int)(w / Hkv), g = heads_outer ? (int)(w / n_blocks) : (int)(w % Hkv);
  int b = 0;
  for (int hi = ct.n_req; hi - b > 1;) { const int mid = (b + hi) >> 1; if (ct.blk_cu[mid] <= x) b = mid; else hi = mid; }
  const long long first = (long long)(x - ct.blk_cu[b]) * block_size;
  const int n = (int)min((long long)block_size, ct.ctx_len[b] - first);
  const uint16_t* p = k + (ct.tok_off[b] + first) * token_stride + g * head_stride + gl * 8;
  uint32_t mx[4], mn[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) { mx[e] = 0x7fff7fffu; mn[e] = 0x7fff7fffu; }       // NaN: passed over by both
  for (int t0 = 0; t0 < n; t0 += U * kTok) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * kTok + sub;
      v[u] = t < n ? *reinterpret_cast<const uint4*>(p + t * token_stride) : make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      mx[0] = bmax2(mx[0], v[u].x); mx[1] = bmax2(mx[1], v[u].y); mx[2] = bmax2(mx[2], v[u].z); mx[3] = bmax2(mx[3], v[u].w);
      mn[0] = bmin2(mn[0], v[u].x); mn[1] = bmin2(mn[1], v[u].y); mn[2] = bmin2(mn[2], v[u].z); mn[3] = bmin2(mn[3], v[u].w);
    }
  }
#pragma unroll
  for (int o = kLanes; o < 32; o <<= 1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mx[e] = bmax2(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], o));
      mn[e] = bmin2(mn[e], __shfl_xor_sync(0xffffffffu, mn[e], o));
    }
  }
  // the largest magnitude among all dims (NaN, where a dim has nothing else, counts as 0)
  uint32_t amax = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      const uint32_t m1 = (mx[e] >> h) & 0x7fffu, m2 = (mn[e] >> h) & 0x7fffu;
      if (m1 <= 0x7f80u) amax = max(amax, m1);
      if (m2 <= 0x7f80u) amax = max(amax, m2);
    }
  }
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  const int ex = scale_exponent(min(amax, 0x7f7fu));               // an infinity is clamped below
  const float inv = power_of_two(-ex);                             // ex <= 122
  auto quantise = [&](uint32_t bits, bool up) -> uint32_t {
    const float f = bf16_bits_to_float((uint16_t)bits) * inv;      // exact, or below the smallest normal number times a power of two
    const float r = up ? ceilf(f) : floorf(f);
    return (uint32_t)(uint8_t)(int8_t)(int)fminf(fmaxf(r, -127.f), 127.f);
  };
  if (sub == 0) {
    uint32_t hi[2] = {0u, 0u}, lo[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t bh = (mx[e >> 1] >> ((e & 1) * 16)) & 0xffffu, bl = (mn[e >> 1] >> ((e & 1) * 16)) & 0xffffu;
      hi[e >> 2] |= ((bh & 0x7fffu) > 0x7f80u ? 0u : quantise(bh, true)) << ((e & 3) * 8);
      lo[e >> 2] |= ((bl & 0x7fffu) > 0x7f80u ? 0u : quantise(bl, false)) << ((e & 3) * 8);
    }
    int8_t* o = bounds + ((long long)x * Hkv + g) * (2 * D) + gl * 8;
    *reinterpret_cast<uint2*>(o) = make_uint2(hi[0], hi[1]);
    *reinterpret_cast<uint2*>(o + D) = make_uint2(lo[0], lo[1]);
    if (gl == 0) scale[(long long)x * Hkv + g] = power_of_two(ex);
  }
}

// ---- scores ---------------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ void mma_s8_16832(int* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

struct SelectArgs {
  const int8_t* bounds;
  const float* scale;
  const uint16_t* q;
  const int *row_cu, *row_seq;
  float* scores;                       // [n_rows, H_kv, most]
  int* out;                            // [n_rows, H_kv, n_select]
  long long n_rows;
  int most, H, Hkv, n_seq, block_size, n_select, n_first, n_last;
};

// Rows of context b in the step; n < 0: more than the host's bounds.
struct RowRange { long long first; int n; };
__device__ __forceinline__ RowRange rows_of(const SelectArgs& a, const ContTable& ct, int b) {
  const long long r0 = a.row_cu[ct.seq_cu[b]], r1 = a.row_cu[ct.seq_cu[b + 1]];
  if (r0 < 0 || r1 < r0 || r1 > a.n_rows || r1 - r0 > ct.max_rows[b]) return {0, -1};
  return {r0, (int)(r1 - r0)};
}

constexpr int kScoWarps = 4;
constexpr int kScoPass = 8;             // row tiles whose queries a block holds at once

// A block: eight context blocks per warp, one KV head, all rows of the context.  PAIR: two rows of the step to an MMA (groups of up to eight heads).
template <int D, bool PAIR>
__global__ void __launch_bounds__(kScoWarps * 32)
block_score_kernel(const __grid_constant__ ContTable ct, const __grid_constant__ SelectArgs a, DeviceStatus* st) {
  constexpr int kSteps = 2 * D / 32;                                // MMAs of a product
  constexpr int kRowsPer = PAIR ? 2 : 1;                            // rows of the step per tile
  __shared__ __align__(16) uint32_t q_s[kScoPass][16][2 * D / 4 + 4];      // [tile][fragment row][q+ | q-]; the rows 16 bytes apart from whole banks
  __shared__ float sq_s[kScoPass][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const int G = a.H / a.Hkv;
  const int hd = blockIdx.y;
  int b = 0;
  for (int hi = ct.n_req; hi - b > 1;) { const int mid = (b + hi) >> 1; if (ct.tile_cu[mid] <= (int)blockIdx.x) b = mid; else hi = mid; }
  const int nb = ct.blk_cu[b + 1] - ct.blk_cu[b], x0 = (((int)blockIdx.x - ct.tile_cu[b]) * kScoWarps + warp) * 8;
  griddep_launch();
  griddep_wait();
  // this lane's share of its block's 2 D bytes: bytes [tig D / 2, + D / 2)
  const int x = x0 + gid;
  uint32_t bd[D / 8];
  {
    const uint4* p = reinterpret_cast<const uint4*>(a.bounds + ((long long)(ct.blk_cu[b] + min(x, nb - 1)) * a.Hkv + hd) * (2 * D) + tig * (D / 2));
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const uint4 v = p[i];
      bd[4 * i] = v.x; bd[4 * i + 1] = v.y; bd[4 * i + 2] = v.z; bd[4 * i + 3] = v.w;
    }
  }
  float sb[2];                                                       // scales of the blocks of this lane's result columns
#pragma unroll
  for (int e = 0; e < 2; ++e) sb[e] = a.scale[(long long)(ct.blk_cu[b] + min(x0 + 2 * tig + e, nb - 1)) * a.Hkv + hd];
  // (the bounds are on their way)
  const RowRange rr = rows_of(a, ct, b);
  if (rr.n < 0 && threadIdx.x == 0 && hd == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_SELECT_BLOCKS, b, ct.max_rows[b]);
  if (rr.n <= 0) return;
  const int n_tiles = (rr.n + kRowsPer - 1) / kRowsPer;
  for (int p0 = 0; p0 < n_tiles; p0 += kScoPass) {
    const int here = min(kScoPass, n_tiles - p0);
    __syncthreads();
    // queries in 8 bits: eight lanes per fragment row, D / 8 dims each, the loads of four steps side by side
    constexpr int kVec = D / 64, kStep = 4 * kScoWarps, kBatch = 4;
    const int ql = lane & 7, sub = lane >> 3;
    for (int i0 = warp * 4 + sub; i0 < here * 16; i0 += kStep * kBatch) {
      uint4 raw[kBatch][kVec];
      bool live[kBatch];
#pragma unroll
      for (int c = 0; c < kBatch; ++c) {
        const int i = i0 + c * kStep, tile = i >> 4, fr = i & 15, r = (p0 + tile) * kRowsPer + (PAIR ? fr >> 3 : 0), h = PAIR ? fr & 7 : fr;
        live[c] = i < here * 16 && h < G && r < rr.n;
        const uint4* p = reinterpret_cast<const uint4*>(a.q + ((rr.first + r) * a.H + hd * G + h) * D + ql * (D / 8));
#pragma unroll
        for (int e = 0; e < kVec; ++e) raw[c][e] = live[c] ? p[e] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int c = 0; c < kBatch; ++c) {
        const int i = i0 + c * kStep, tile = i >> 4, fr = i & 15;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(raw[c]);
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < 4 * kVec; ++e) {
#pragma unroll
          for (int hf = 0; hf < 32; hf += 16) {
            const uint32_t m = (w[e] >> hf) & 0x7fffu;
            amax = max(amax, m <= 0x7f80u ? m : 0u);
          }
        }
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        const int ex = scale_exponent(min(amax, 0x7f7fu));
        const float inv = power_of_two(-ex);
        uint32_t pos[2 * kVec], neg[2 * kVec];
#pragma unroll
        for (int e = 0; e < 2 * kVec; ++e) {
          pos[e] = neg[e] = 0u;
#pragma unroll
          for (int b4 = 0; b4 < 4; ++b4) {
            const uint32_t bits = (w[2 * e + (b4 >> 1)] >> ((b4 & 1) * 16)) & 0xffffu;
            const float f = (bits & 0x7fffu) > 0x7f80u ? 0.f : rintf(bf16_bits_to_float((uint16_t)bits) * inv);
            pos[e] |= (uint32_t)(int)fminf(fmaxf(f, 0.f), 127.f) << (b4 * 8);
            neg[e] |= ((uint32_t)(int)fmaxf(fminf(f, 0.f), -127.f) & 0xffu) << (b4 * 8);
          }
        }
        if (i < here * 16) {
          uint32_t* row = q_s[tile][fr];
#pragma unroll
          for (int e = 0; e < 2 * kVec; ++e) {
            row[ql * 2 * kVec + e] = pos[e];
            row[D / 4 + ql * 2 * kVec + e] = neg[e];
          }
          if (ql == 0) sq_s[tile][fr] = live[c] ? power_of_two(ex) : -1.f;      // no such row or head
        }
      }
    }
    __syncthreads();
    if (x0 >= nb) continue;
    for (int tile = 0; tile < here; ++tile) {
      int acc[4] = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const uint2 qa = *reinterpret_cast<const uint2*>(&q_s[tile][gid][tig * (D / 8) + 2 * s]);
        const uint2 qb = *reinterpret_cast<const uint2*>(&q_s[tile][gid + 8][tig * (D / 8) + 2 * s]);
        const uint32_t fa[4] = {qa.x, qb.x, qa.y, qb.y};
        mma_s8_16832(acc, fa, bd[2 * s], bd[2 * s + 1]);
      }
      // the largest over the heads of a row: fragment rows lie 4 lanes apart
      float best[2][2];
      const float s0 = sq_s[tile][gid], s1 = sq_s[tile][gid + 8];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        best[0][e] = s0 > 0.f ? (float)acc[e] * s0 : -INFINITY;
        best[1][e] = s1 > 0.f ? (float)acc[2 + e] * s1 : -INFINITY;
        if (!PAIR) best[0][e] = fmaxf(best[0][e], best[1][e]);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          best[0][e] = fmaxf(best[0][e], __shfl_xor_sync(0xffffffffu, best[0][e], o));
          if (PAIR) best[1][e] = fmaxf(best[1][e], __shfl_xor_sync(0xffffffffu, best[1][e], o));
        }
      }
      if (gid < kRowsPer) {
        const int r = (p0 + tile) * kRowsPer + gid;
        if (r < rr.n) {
          float* o = a.scores + ((rr.first + r) * a.Hkv + hd) * a.most;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int xx = x0 + 2 * tig + e;
            if (xx < nb) o[xx] = best[gid][e] * sb[e] + 0.f;                     // (+ 0: one zero, not two)
          }
        }
      }
    }
  }
}

// ---- the n_select highest scores of a (row, KV head) ------------------------------------------------------------------------------

constexpr int kTopThreads = 256;
constexpr int kTopKept = 8192;          // scores that a block keeps in shared memory; more are read again by every pass
constexpr int kTopBits = 10;

// Order-preserving key of a score (no NaN: scores are products of whole numbers and powers of two).
__device__ __forceinline__ uint32_t score_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The first and last blocks are taken in any case; of the others the `want` highest.  Their keys' common leading bits are skipped, then digits of ten
// bits are counted from the highest on until the digit that the want-th key falls into holds no more keys than are wanted: with spread scores
// two counts.  A launch of few rows is a chain of latencies and barriers.
__global__ void __launch_bounds__(kTopThreads)
block_topk_kernel(const __grid_constant__ ContTable ct, const __grid_constant__ SelectArgs a, DeviceStatus* st) {
  constexpr int kBins = 1 << kTopBits, kBinsPer = kBins / kTopThreads, kWarps = kTopThreads / 32, U = 8;
  extern __shared__ uint32_t key_s[];
  __shared__ int hist[kBins];
  __shared__ int warp_sum[kWarps], found[2];
  __shared__ uint2 warp_range[kWarps];
  __shared__ int2 warp_pair[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int hd = (int)(blockIdx.x % a.Hkv);
  const long long row = blockIdx.x / a.Hkv;
  // (No early call for the next kernel: the attention's clusters, placed while these blocks are still there, ran 6 us longer, 29.4 / 35.8 for a
  // pass over four rows of 32 K.)
  griddep_wait();
  const int seq = a.row_seq[row];
  if (seq == -1) return;
  if (seq < 0 || seq >= a.n_seq) {
    if (tid == 0 && hd == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_SELECT_BLOCKS, seq, (int)row);
    return;
  }
  const int b = context_of(ct, seq), nb = ct.blk_cu[b + 1] - ct.blk_cu[b];
  const RowRange rr = rows_of(a, ct, b);
  const float* score = a.scores + (row * a.Hkv + hd) * a.most;
  int* out = a.out + (row * a.Hkv + hd) * a.n_select;
  const bool mine = rr.n >= 0 && row >= rr.first && row < rr.first + rr.n;
  if (!mine && tid == 0 && hd == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_SELECT_BLOCKS, (int)row, b);
  if (nb <= a.n_select) {                                                        // all of them
    for (int i = tid; mine && i < a.n_select; i += kTopThreads) out[i] = i < nb ? i : -1;
    return;
  }
  const int x0 = a.n_first, x1 = nb - a.n_last;                                  // blocks that compete: [x0, x1), more than are wanted
  const bool kept = nb <= kTopKept;
  uint32_t lo = 0xffffffffu, hi = 0u;
  for (int i0 = x0 + tid; i0 < x1; i0 += U * kTopThreads) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = i0 + u * kTopThreads < x1 ? score[i0 + u * kTopThreads] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kTopThreads;
      if (i < x1) {
        const uint32_t k = score_key(v[u]);
        if (kept) key_s[i] = k;
        lo = min(lo, k);
        hi = max(hi, k);
      }
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) warp_range[warp] = make_uint2(lo, hi);
  for (int i = tid; i < kBins; i += kTopThreads) hist[i] = 0;
  if (!mine) return;                                                             // (the whole block)
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) { lo = min(lo, warp_range[w].x); hi = max(hi, warp_range[w].y); }
  auto key_of = [&](int i) -> uint32_t { return kept ? key_s[i] : score_key(score[i]); };
  int want = a.n_select - a.n_first - a.n_last;                                  // of the keys in [base, base + 2^left), the want-th highest is looked for
  int left = 32 - __clz(lo ^ hi);                                                // bits that are not common
  uint32_t base = left >= 32 ? 0u : lo >> left << left;
  bool all_in = false;                                                           // every key from base on is taken: no ties to break
  if (want == 0) { base = 0xffffffffu; all_in = true; left = 0; }
  while (left > 0) {
    const int shift = max(0, left - kTopBits);
    for (int i = x0 + tid; i < x1; i += kTopThreads) {
      const uint32_t d = key_of(i) - base;
      if (left >= 32 || (d >> left) == 0) atomicAdd(&hist[d >> shift], 1);       // (keys below base wrap round and fall out)
    }
    __syncthreads();
    // bins from the highest: thread t has bins (top - kBinsPer (t + 1), top - kBinsPer t]
    int cnt[kBinsPer], mine_n = 0;
#pragma unroll
    for (int e = 0; e < kBinsPer; ++e) {
      const int bin = kBins - 1 - tid * kBinsPer - e;
      cnt[e] = hist[bin];
      hist[bin] = 0;
      mine_n += cnt[e];
    }
    int incl = mine_n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int before = incl - mine_n;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    if (before < want && before + mine_n >= want) {                              // exactly one thread
#pragma unroll
      for (int e = 0; e < kBinsPer; ++e) {
        if (before < want && before + cnt[e] >= want) {
          found[0] = (kBins - 1 - tid * kBinsPer - e) | (before + cnt[e] == want ? 1 << 30 : 0);
          found[1] = want - before;
        }
        before += cnt[e];
      }
    }
    __syncthreads();
    base += (uint32_t)(found[0] & ((1 << 30) - 1)) << shift;
    want = found[1];
    left = shift;
    if (found[0] >> 30) { all_in = true; break; }
    __syncthreads();
  }
  // ---- keys above, and of those equal to base the first `want`: every thread a range in order ----
  const int per = (nb + kTopThreads - 1) / kTopThreads, i0 = min(nb, tid * per), i1 = min(nb, i0 + per);
  auto kind = [&](int i) -> int {                                                // 2: taken, 1: equal to the last one, 0: left
    if (i < x0 || i >= x1) return 2;
    const uint32_t k = key_of(i);
    return all_in ? (k >= base ? 2 : 0) : k > base ? 2 : k == base ? 1 : 0;
  };
  int above = 0, equal = 0;
  for (int i = i0; i < i1; ++i) { const int k = kind(i); above += k == 2; equal += k == 1; }
  int ia = above, ie = equal;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int va = __shfl_up_sync(0xffffffffu, ia, o), ve = __shfl_up_sync(0xffffffffu, ie, o);
    if (lane >= o) { ia += va; ie += ve; }
  }
  if (lane == 31) warp_pair[warp] = make_int2(ia, ie);
  __syncthreads();
  ia -= above; ie -= equal;
  for (int w = 0; w < warp; ++w) { ia += warp_pair[w].x; ie += warp_pair[w].y; }
  if (all_in) want = 0;
  int at = ia + min(ie, want);
  for (int i = i0; i < i1; ++i) {
    const int k = kind(i);
    if (k == 2 || (k == 1 && ie++ < want)) out[at++] = i;
  }
}

}  // namespace relaxkv

using namespace relaxkv;

extern "C" relaxkv_status relaxkv_block_bounds(const relaxkv_shape* shape, const relaxkv_cache_view* cache, int32_t block_size, int8_t* bounds_out,
                                               float* scale_out, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_block_bounds");
  relaxkv_status rc = check_contexts(shape);
  if (rc != RELAXKV_OK) return rc;
  if (!block_size_ok(block_size)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  long long blocks = 0;
  for (int b = 0; b < shape->n_req; ++b) blocks += ((long long)shape->h_ctx_len[b] + block_size - 1) / block_size;
  if (blocks == 0) return RELAXKV_OK;
  if ((rc = check_cache(shape, cache, false)) != RELAXKV_OK) return rc;
  if (!bounds_out || !scale_out || !aligned16(bounds_out)) return RELAXKV_ERR_INVALID_ARG;
  const int Hkv = shape->n_kv_heads, D = shape->head_dim;
  if (blocks * Hkv > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  ContTable ct;
  fill_contexts(ct, shape, cache, block_size);
  const unsigned grid = (unsigned)((blocks * Hkv + kBndThreads / 32 - 1) / (kBndThreads / 32));
  auto kern = D == 128 ? block_bounds_kernel<128> : block_bounds_kernel<64>;
  return cuda_ok(launch_chained(kern, dim3(grid), kBndThreads, 0, static_cast<cudaStream_t>(stream), static_cast<const uint16_t*>(cache->k),
                                (long long)cache->token_stride, (long long)cache->head_stride, ct, block_size, Hkv, bounds_out, scale_out,
                                cache->head_stride > cache->token_stride ? 1 : 0));
}

extern "C" relaxkv_status relaxkv_select_blocks(
    const relaxkv_shape* shape, int32_t block_size, const int8_t* bounds, const float* scale, const relaxkv_continuation_rows* rows, const void* q,
    int32_t n_select, int32_t n_first, int32_t n_last, int32_t* blocks_out, void* workspace, size_t workspace_bytes, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_select_blocks");
  relaxkv_status rc = check_contexts(shape);
  if (rc != RELAXKV_OK) return rc;
  if (!block_size_ok(block_size)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (n_select < 1 || n_first < 0 || n_last < 0 || (long long)n_first + n_last > n_select) return RELAXKV_ERR_INVALID_ARG;
  ContTable ct;
  long long blocks = 0;
  for (int b = 0; b < shape->n_req; ++b) blocks += ((long long)shape->h_ctx_len[b] + block_size - 1) / block_size;
  if (blocks * shape->n_kv_heads > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  fill_contexts(ct, shape, nullptr, block_size);
  if ((rc = check_rows(shape, rows, false, ct)) != RELAXKV_OK) return rc;
  if (!q || !aligned16(q) || !blocks_out || !workspace || (blocks > 0 && (!bounds || !scale || !aligned16(bounds)))) return RELAXKV_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return RELAXKV_ERR_INVALID_ARG;
  if (workspace_bytes < cont_ws(shape, rows->n_rows, block_size).total) return RELAXKV_ERR_WORKSPACE_TOO_SMALL;
  if (rows->n_rows == 0) return RELAXKV_OK;
  if (rows->n_rows * shape->n_kv_heads > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  DeviceStatus* st = status_word();
  if (!st) return RELAXKV_ERR_CUDA;
  SelectArgs a = {};
  a.bounds = bounds; a.scale = scale; a.q = static_cast<const uint16_t*>(q);
  a.row_cu = rows->row_cu; a.row_seq = rows->row_seq;
  a.scores = static_cast<float*>(workspace); a.out = blocks_out; a.n_rows = rows->n_rows;
  a.H = shape->n_q_heads; a.Hkv = shape->n_kv_heads; a.n_seq = rows->n_seq; a.block_size = block_size;
  a.n_select = n_select; a.n_first = n_first; a.n_last = n_last;
  for (int b = 0; b < ct.n_req; ++b) {
    const int nb = ct.blk_cu[b + 1] - ct.blk_cu[b];
    a.most = std::max(a.most, nb);
    // contexts of no more blocks than are selected need no scores
    ct.tile_cu[b + 1] = ct.tile_cu[b] + (nb > n_select && ct.max_rows[b] > 0 ? (nb + 8 * kScoWarps - 1) / (8 * kScoWarps) : 0);
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int D = shape->head_dim;
  if (a.Hkv > 65535) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (ct.tile_cu[ct.n_req] > 0) {
    const bool pair = a.H / a.Hkv <= 8;
    auto kern = D == 128 ? (pair ? block_score_kernel<128, true> : block_score_kernel<128, false>)
                         : (pair ? block_score_kernel<64, true> : block_score_kernel<64, false>);
    rc = cuda_ok(launch_chained(kern, dim3((unsigned)ct.tile_cu[ct.n_req], (unsigned)a.Hkv), kScoWarps * 32, 0, s, ct, a, st));
    if (rc != RELAXKV_OK) return rc;
  }
  const size_t smem = a.most <= kTopKept ? (size_t)a.most * 4 : 0;
  return cuda_ok(launch_chained(block_topk_kernel, dim3((unsigned)(a.n_rows * a.Hkv)), kTopThreads, smem, s, ct, a, st));
}
