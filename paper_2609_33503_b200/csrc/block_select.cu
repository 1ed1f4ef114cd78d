// Context blocks by a cheap score: 8-bit bounds of every block's keys (relaxkv_block_bounds), and the blocks of the highest score for each row
// and KV head (relaxkv_select_blocks): the largest logit of a key within the bounds, of the query as it is in 8 bits.
//
// Bounds: one pass over K, bound by its bytes.  A warp has one (block, KV head): 16 lanes hold the 128 dims of a token as 16-byte pieces, so
// a load takes two tokens (four of 64 dims); maxima and minima stay packed bf16 pairs and are exact.  The scale is a power of two, so are the
// quotients, and the rounding is away from the block: the bounds remain bounds (but for infinite keys, which are clamped).  The query is rounded to
// the nearest number, so a score may lie below a logit of the query itself.
// Scores: sum_d max(q_d hi_d, q_d lo_d) = q+ . hi + q- . lo, a product over 2 D whole numbers of 8 bits, as halves on the tensor cores with sums in
// 32 bits: rows are the heads of one, two or four rows of the step, columns eight blocks.  All are whole numbers below 2^24, so the scores, and with them
// the lists, do not depend on the order of anything; it may be any as long as both sides agree, so a lane takes D / 2 bytes of its block in
// 16-byte loads and the queries are laid out to match.  Up to four tiles of rows go to a block, so that rows and context blocks both spread
// over the SMs: with all rows in one block, 64 rows of 40 / 8 heads over 938 blocks took 33 us, so 27 (24.5 by now).
// Selection: one block per (row, KV head); counts of digits find the lowest selected score, then every warp writes its own range's blocks in
// order.  Both launches: 4 rows of 40 / 8 heads, 512 blocks 8.0 us, 16 rows of 32 / 8 heads in two contexts of some 2000 blocks 13.6: latencies
// (row -> query -> product -> score -> counts), not bytes; 64 rows in one context of 8192 blocks 81.
#include "continuation_splits.cuh"
#include "continuations.cuh"
#include <algorithm>
#include <cuda_fp16.h>

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

// U: loads of a lane that travel together, 16 where a block has as many.  Blocks of 64 tokens, 8 heads of 128 dims: 16 K tokens (33.5 MB) 7.2 us,
// 131 K (268 MB) 43.6 = 6.2 TB/s, with eight loads 9.7 and 44.4; blocks of 16 tokens, 16 K: 8.8 with eight, 11.7 with sixteen, half of them empty.
template <int D, int U>
__global__ void __launch_bounds__(kBndThreads)
block_bounds_kernel(const uint16_t* k, long long token_stride, long long head_stride, const __grid_constant__ ContTable ct, int block_size, int Hkv,
                    int8_t* bounds, float* scale, int heads_outer) {
  constexpr int kLanes = D / 8, kTok = 32 / kLanes;
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

__device__ __forceinline__ void mma_f16_16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }
// Four whole numbers of 8 bits as halves: with 128 added, a byte behind 0x64 is the half 1024 + byte.
__device__ __forceinline__ void halves_of(uint32_t bytes, uint32_t* h) {
  const uint32_t u = bytes ^ 0x80808080u, lo = __byte_perm(u, 0x64646464u, 0x4140), hi = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 off = __float2half2_rn(1152.f);
  h[0] = h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&lo), off));
  h[1] = h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&hi), off));
}

struct SelectArgs {
  const int8_t* bounds;
  const float* scale;
  const uint16_t* q;
  const int *row_cu, *row_seq;
  float* scores;                       // [n_rows, H_kv, most]
  int* out;                            // [n_rows, H_kv, n_select]
  long long n_rows;
  int most, H, Hkv, n_seq, n_select, n_first, n_last;
  int kept;                            // scores that a block of the selection has shared memory for
};

// Rows of context b in the step; n < 0: more than the host's bounds.
struct RowRange { long long first; int n; };
__device__ __forceinline__ RowRange rows_of(const SelectArgs& a, const ContTable& ct, int b) {
  const long long r0 = a.row_cu[ct.seq_cu[b]], r1 = a.row_cu[ct.seq_cu[b + 1]];
  if (r0 < 0 || r1 < r0 || r1 > a.n_rows || r1 - r0 > ct.max_rows[b]) return {0, -1};
  return {r0, (int)(r1 - r0)};
}

constexpr int kScoWarps = 4;
constexpr int kScoCols = 2;             // times eight context blocks of a warp
constexpr int kScoPass = 4;             // row tiles of a block

// A block: sixteen context blocks per warp, one KV head, up to kScoPass tiles of the context's rows.  ROWS: rows of the step to an MMA, 16 / ROWS heads of each.
template <int D, int ROWS>
__global__ void __launch_bounds__(kScoWarps * 32)
block_score_kernel(const __grid_constant__ ContTable ct, const __grid_constant__ SelectArgs a, DeviceStatus* st) {
  constexpr int kSteps = 2 * D / 16;                                // MMAs of a product
  constexpr int kHeads = 16 / ROWS;                                 // fragment rows of a row of the step
  __shared__ __align__(16) uint32_t q_s[kScoPass][16][D + 8];       // [tile][fragment row][step, in an order][lane of four] four halves of (q+ | q-)
  __shared__ float sq_s[kScoPass][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const int G = a.H / a.Hkv;
  const int hd = blockIdx.y;
  int b = 0;
  for (int hi = ct.n_req; hi - b > 1;) { const int mid = (b + hi) >> 1; if (ct.tile_cu[mid] <= (int)blockIdx.x) b = mid; else hi = mid; }
  const int nb = ct.blk_cu[b + 1] - ct.blk_cu[b], across = (nb + 8 * kScoCols * kScoWarps - 1) / (8 * kScoCols * kScoWarps);
  const int p0 = ((int)blockIdx.x - ct.tile_cu[b]) / across * kScoPass;
  const int x0 = (((int)blockIdx.x - ct.tile_cu[b]) % across * kScoWarps + warp) * (8 * kScoCols);
  griddep_launch();
  griddep_wait();
  // this lane's share of its blocks' 2 D bytes: bytes [tig D / 2, + D / 2) of block x0 + gid (and of the eight behind)
  uint4 bytes[kScoCols][D / 32];
  float sb[kScoCols][2];                                             // scales of the blocks of this lane's result columns
#pragma unroll
  for (int c = 0; c < kScoCols; ++c) {
    const uint4* p = reinterpret_cast<const uint4*>(a.bounds + ((long long)(ct.blk_cu[b] + min(x0 + 8 * c + gid, nb - 1)) * a.Hkv + hd) * (2 * D) + tig * (D / 2));
#pragma unroll
    for (int i = 0; i < D / 32; ++i) bytes[c][i] = p[i];
#pragma unroll
    for (int e = 0; e < 2; ++e) sb[c][e] = a.scale[(long long)(ct.blk_cu[b] + min(x0 + 8 * c + 2 * tig + e, nb - 1)) * a.Hkv + hd];
  }
  // (the bounds are on their way)
  const RowRange rr = rows_of(a, ct, b);
  if (rr.n < 0 && threadIdx.x == 0 && hd == 0 && p0 == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_SELECT_BLOCKS, b, ct.max_rows[b]);
  const int here = min(kScoPass, (rr.n + ROWS - 1) / ROWS - p0);
  if (rr.n < 0 || here <= 0) return;
  // queries in 8 bits: eight lanes per fragment row, D / 8 dims each, all loads side by side
  constexpr int kVec = D / 64, kStep = 4 * kScoWarps, kBatch = 16 * kScoPass / kStep;
  const int ql = lane & 7, sub = lane >> 3;
  uint4 raw[kBatch][kVec];
  bool live[kBatch];
#pragma unroll
  for (int c = 0; c < kBatch; ++c) {
    const int i = warp * 4 + sub + c * kStep, tile = i >> 4, fr = i & 15, r = (p0 + tile) * ROWS + fr / kHeads, h = fr % kHeads;
    live[c] = i < here * 16 && h < G && r < rr.n;
    const uint4* p = reinterpret_cast<const uint4*>(a.q + ((rr.first + r) * a.H + hd * G + h) * D + ql * (D / 8));
#pragma unroll
    for (int e = 0; e < kVec; ++e) raw[c][e] = live[c] ? p[e] : make_uint4(0u, 0u, 0u, 0u);
  }
  uint32_t bd[kScoCols][D / 4];
#pragma unroll
  for (int c = 0; c < kScoCols; ++c) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      halves_of(bytes[c][i].x, &bd[c][8 * i]);
      halves_of(bytes[c][i].y, &bd[c][8 * i + 2]);
      halves_of(bytes[c][i].z, &bd[c][8 * i + 4]);
      halves_of(bytes[c][i].w, &bd[c][8 * i + 6]);
    }
  }
#pragma unroll
  for (int c = 0; c < kBatch; ++c) {
    const int i = warp * 4 + sub + c * kStep, tile = i >> 4, fr = i & 15;
    if (i >= here * 16) break;                        // (the same for a warp's lanes)
    if (ql == 0 && !live[c]) sq_s[tile][fr] = -1.f;   // no such row or head: its scores are passed over, whatever they are
    if (!__any_sync(0xffffffffu, live[c])) continue;
    const uint32_t* w = reinterpret_cast<const uint32_t*>(raw[c]);
    uint32_t top = w[0] & 0x7fff7fffu;
#pragma unroll
    for (int e = 1; e < 4 * kVec; ++e) top = bmax2(top, w[e] & 0x7fff7fffu);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) top = bmax2(top, __shfl_xor_sync(0xffffffffu, top, o));
    // the larger half; NaN is left only where there is nothing else
    const uint32_t t0 = top & 0xffffu, t1 = top >> 16, amax = max(t0 > 0x7f80u ? 0u : t0, t1 > 0x7f80u ? 0u : t1);
    const int ex = scale_exponent(min(amax, 0x7f7fu));
    const float inv = power_of_two(-ex);
    // to the nearest whole number, ties to the even one; NaN is neither above nor below zero
    uint2* row = reinterpret_cast<uint2*>(q_s[tile][fr]);
    constexpr float kWhole = 12582912.f;
    const __half2 zero = __float2half2_rn(0.f), most = __float2half2_rn(127.f), least = __float2half2_rn(-127.f);
#pragma unroll
    for (int e = 0; e < 2 * kVec; ++e) {
      uint32_t pos[2], neg[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint32_t bits = w[2 * e + u];
        const __half2 v = __floats2half2_rn((__uint_as_float(bits << 16) * inv + kWhole) - kWhole, (__uint_as_float(bits & 0xffff0000u) * inv + kWhole) - kWhole);
        pos[u] = h2_bits(__hmin2(__hmax2(v, zero), most));
        neg[u] = h2_bits(__hmax2(__hmin2(v, zero), least));
      }
      const int at = (4 * e + (ql & 3)) * 4 + (ql >> 2);                  // step 2 kVec (ql & 3) + e, lane of the four: steps apart by banks
      row[at] = make_uint2(pos[0], pos[1]);
      row[at + 2] = make_uint2(neg[0], neg[1]);
    }
    if (ql == 0 && live[c]) sq_s[tile][fr] = power_of_two(ex);
  }
  __syncthreads();
  if (x0 >= nb) return;
  for (int tile = 0; tile < here; ++tile) {
    // (sums of an even and an odd half of the steps, so that they need not wait for each other)
    float acc[kScoCols][2][4];
#pragma unroll
    for (int c = 0; c < kScoCols; ++c) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[c][0][e] = acc[c][1][e] = 0.f;
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int at = 8 * (s % (2 * kVec) * 4 + s / (2 * kVec)) + 2 * tig;
      const uint2 qa = *reinterpret_cast<const uint2*>(&q_s[tile][gid][at]);
      const uint2 qb = *reinterpret_cast<const uint2*>(&q_s[tile][gid + 8][at]);
#pragma unroll
      for (int c = 0; c < kScoCols; ++c) mma_f16_16816(acc[c][s & 1], qa.x, qb.x, qa.y, qb.y, bd[c][2 * s], bd[c][2 * s + 1]);
    }
    // the largest over the heads of a row, whose fragment rows lie 4 lanes apart: of the values (half of the fragment rows, column tile, column)
    // a lane keeps one side of each in turn and hands over the other
    static_assert(kScoCols == 2, "two column tiles");
    float v[8];
    const float s0 = sq_s[tile][gid], s1 = sq_s[tile][gid + 8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float *even = acc[e >> 1][0], *odd = acc[e >> 1][1];
      v[e] = s0 > 0.f ? (even[e & 1] + odd[e & 1]) * s0 : -INFINITY;
      v[4 + e] = s1 > 0.f ? (even[2 + (e & 1)] + odd[2 + (e & 1)]) * s1 : -INFINITY;
      if (ROWS == 1) v[e] = fmaxf(v[e], v[4 + e]);
    }
    int o = 4;
    auto halve = [&](int n) {                                            // of 2 n values, this lane keeps n
      const bool up = (lane & o) != 0;
#pragma unroll
      for (int e = 0; e < n; ++e) {
        const float keep = up ? v[n + e] : v[e], give = up ? v[e] : v[n + e];
        v[e] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, give, o));
      }
      o <<= 1;
    };
    if (ROWS > 1) halve(4);
    halve(2);
    if (ROWS < 4) halve(1);
    if (ROWS == 1) v[0] = fmaxf(v[0], __shfl_xor_sync(0xffffffffu, v[0], 16));
    const int half = ROWS > 1 ? gid & 1 : 0, c = ROWS > 1 ? (gid >> 1) & 1 : gid & 1, r = (p0 + tile) * ROWS + (ROWS == 4 ? 2 * half + (gid >> 2) : half);
    if (r < rr.n && (ROWS > 1 || gid < 4)) {
      float* out = a.scores + ((rr.first + r) * a.Hkv + hd) * a.most;
#pragma unroll
      for (int e = 0; e < (ROWS == 4 ? 2 : 1); ++e) {
        const int col = ROWS == 4 ? e : ROWS == 2 ? gid >> 2 : (gid >> 1) & 1, xx = x0 + 8 * c + 2 * tig + col;
        const float scale = c ? (col ? sb[1][1] : sb[1][0]) : (col ? sb[0][1] : sb[0][0]);
        if (xx < nb) out[xx] = v[e] * scale + 0.f;                        // (+ 0: one zero, not two)
      }
    }
  }
}

// ---- the n_select highest scores of a (row, KV head) ------------------------------------------------------------------------------

constexpr int kTopKept = 8192;          // scores that a block keeps in shared memory, at most; more are read again by every pass

// Order-preserving key of a score (no NaN: scores are products of whole numbers and powers of two).
__device__ __forceinline__ uint32_t score_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The first and last blocks are taken in any case; of the others the `want` highest.  Their keys' common leading bits are skipped, then digits are
// counted from the highest on, a digit's value per thread, until the one that the want-th key falls into holds no more keys than are wanted: with
// spread scores two counts.  A launch of few rows is a chain of latencies and barriers.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
block_topk_kernel(const __grid_constant__ ContTable ct, const __grid_constant__ SelectArgs a, DeviceStatus* st) {
  constexpr int kBits = THREADS > 256 ? 9 : 8, kWarps = THREADS / 32, U = 8;
  extern __shared__ uint32_t key_s[];
  static_assert(THREADS == 1 << kBits, "a bin per thread");
  __shared__ int hist[THREADS];
  __shared__ int warp_sum[kWarps], found[2];
  __shared__ uint2 warp_range[kWarps];
  __shared__ int2 warp_pair[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int hd = (int)(blockIdx.x % a.Hkv);
  const long long row = blockIdx.x / a.Hkv;
  // (No early call for the next kernel: the attention's clusters cannot come to the SMs of these blocks, whose shared memory is set up otherwise, and
  // crowd onto the rest: 36.7 us for a pass over four rows of 32 K.  With the same set-up for all kernels 29.5, like this 29.0.)
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
    for (int i = tid; mine && i < a.n_select; i += THREADS) out[i] = i < nb ? i : -1;
    return;
  }
  const int x0 = a.n_first, x1 = nb - a.n_last;                                  // blocks that compete: [x0, x1), more than are wanted
  const bool kept = nb <= a.kept;                                                // (the launch's shared memory: contexts of a call differ)
  uint32_t lo = 0xffffffffu, hi = 0u;
  for (int i0 = x0 + tid; i0 < x1; i0 += U * THREADS) {
    float v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = i0 + u * THREADS < x1 ? score[i0 + u * THREADS] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * THREADS;
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
  hist[tid] = 0;
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
    const int shift = max(0, left - kBits);
    for (int i = x0 + tid; i < x1; i += THREADS) {
      const uint32_t d = key_of(i) - base;
      if (left >= 32 || (d >> left) == 0) atomicAdd(&hist[d >> shift], 1);       // (keys below base wrap round and fall out)
    }
    __syncthreads();
    // thread t has bin THREADS - 1 - t: the sums run from the highest on
    const int bin = THREADS - 1 - tid, n = hist[bin];
    hist[bin] = 0;
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += v; }
    if (lane == 31) warp_sum[warp] = incl;
    __syncthreads();
    int before = incl - n;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    if (before < want && before + n >= want) {                                   // exactly one thread
      found[0] = bin | (before + n == want ? 1 << 30 : 0);
      found[1] = want - before;
    }
    __syncthreads();
    base += (uint32_t)(found[0] & ((1 << 30) - 1)) << shift;
    want = found[1];
    left = shift;
    if (found[0] >> 30) { all_in = true; break; }
    __syncthreads();
  }
  // ---- keys above, and of those equal to base the first `want`: every warp a range in order, 32 keys at a time ----
  const int per = (nb + 32 * kWarps - 1) / (32 * kWarps) * 32, i0 = min(nb, warp * per), i1 = min(nb, i0 + per);
  auto kind = [&](int i) -> int {                                                // 2: taken, 1: equal to the last one, 0: left
    if (i >= i1) return 0;
    if (i < x0 || i >= x1) return 2;
    const uint32_t k = key_of(i);
    return all_in ? (k >= base ? 2 : 0) : k > base ? 2 : k == base ? 1 : 0;
  };
  int above = 0, equal = 0;
  for (int i = i0; i < i1; i += 32) {
    const int k = kind(i + lane);
    above += __popc(__ballot_sync(0xffffffffu, k == 2));
    equal += __popc(__ballot_sync(0xffffffffu, k == 1));
  }
  if (lane == 0) warp_pair[warp] = make_int2(above, equal);
  __syncthreads();
  int ia = 0, ie = 0;
  for (int w = 0; w < warp; ++w) { ia += warp_pair[w].x; ie += warp_pair[w].y; }
  if (all_in) want = 0;
  int at = ia + min(ie, want);
  const uint32_t lower = (1u << lane) - 1u;
  for (int i = i0; i < i1; i += 32) {
    const int k = kind(i + lane);
    const uint32_t ties = __ballot_sync(0xffffffffu, k == 1);
    const uint32_t taken = __ballot_sync(0xffffffffu, k == 2 || (k == 1 && ie + __popc(ties & lower) < want));
    if ((taken >> lane) & 1u) out[at + __popc(taken & lower)] = i + lane;
    at += __popc(taken);
    ie += __popc(ties);
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
  const bool wide = block_size >= 16 * (256 / D);      // sixteen loads are no more than a block has
  auto kern = D == 128 ? (wide ? block_bounds_kernel<128, 16> : block_bounds_kernel<128, 8>)
                       : (wide ? block_bounds_kernel<64, 16> : block_bounds_kernel<64, 8>);
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
  a.H = shape->n_q_heads; a.Hkv = shape->n_kv_heads; a.n_seq = rows->n_seq;
  a.n_select = n_select; a.n_first = n_first; a.n_last = n_last;
  const int G = a.H / a.Hkv, rows_per = (G <= 4 ? 4 : G <= 8 ? 2 : 1) * kScoPass;
  long long tiles = 0;
  for (int b = 0; b < ct.n_req; ++b) {
    const int nb = ct.blk_cu[b + 1] - ct.blk_cu[b];
    a.most = std::max(a.most, nb);
    // contexts of no more blocks than are selected need no scores
    const long long across = (nb + 8 * kScoCols * kScoWarps - 1) / (8 * kScoCols * kScoWarps);
    tiles += nb > n_select ? across * ((ct.max_rows[b] + rows_per - 1) / rows_per) : 0;
    if (tiles > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
    ct.tile_cu[b + 1] = (int)tiles;
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int D = shape->head_dim;
  if (a.Hkv > 65535) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (ct.tile_cu[ct.n_req] > 0) {
    auto kern = D == 128 ? (G <= 4 ? block_score_kernel<128, 4> : G <= 8 ? block_score_kernel<128, 2> : block_score_kernel<128, 1>)
                         : (G <= 4 ? block_score_kernel<64, 4> : G <= 8 ? block_score_kernel<64, 2> : block_score_kernel<64, 1>);
    rc = cuda_ok(launch_chained(kern, dim3((unsigned)ct.tile_cu[ct.n_req], (unsigned)a.Hkv), kScoWarps * 32, 0, s, ct, a, st));
    if (rc != RELAXKV_OK) return rc;
  }
  a.kept = kept_scores(ct.blk_cu, ct.n_req, n_select, kTopKept);
  const size_t smem = (size_t)a.kept * 4;
  const bool many = a.most > 1024;
  auto kern = many ? block_topk_kernel<512> : block_topk_kernel<256>;
  return cuda_ok(launch_chained(kern, dim3((unsigned)(a.n_rows * a.Hkv)), many ? 512 : 256, smem, s, ct, a, st));
}
