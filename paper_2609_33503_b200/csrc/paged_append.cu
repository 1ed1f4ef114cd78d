// Head norm, rotary embedding and append to the paged store of a step's rows in one pass (relaxkv_qk_norm_rope_append_paged).
//
// Reads Q, K, V once and writes rotated Q and the store's K and V once: bound by HBM for many rows and by its latencies (row values, then slot) for
// few.  D / 8 lanes hold one head, each four dims of its first half and the four that they are rotated with, as two 8-byte pieces: the pair
// meets in one lane, and a warp works on two heads of 128 dims (four of 64) at once.  All heads of a row turn by the same angles, so a lane keeps
// its four (cos, sin) in registers; they are made once per row, one angle per thread in double precision, while the first heads are on their
// way.  (With 16-byte pieces, the partner in another lane and the angles read from shared memory for every head, 8205 rows of 40 / 8 heads of 128 with
// norms took 101 us, bound by shared memory.)  Now 49 us = 4.8 TB/s.  Two heads per group of lanes are on their way while two are worked on, and four
// blocks share an SM: with four heads and three blocks 53 us, with one and six 78.  Values stay in fp32 from the load to the one rounding at the
// store.
#include "continuations.cuh"

namespace relaxkv {

constexpr int kPapThreads = 256, kPapAhead = 2;

struct PagedAppendArgs {
  const uint16_t *q, *k, *v, *wq, *wk;
  uint16_t *q_out, *store_k, *store_v;
  const int *positions, *slots;
  long long block_stride, token_stride, head_stride, n_rows;
  int n_blocks, block_shift, H, Hkv;
  float eps;
  double log2_theta;
};

__device__ __forceinline__ void unpack_4(const uint2& r, float* f) {
  f[0] = __uint_as_float(r.x << 16); f[1] = __uint_as_float(r.x & 0xffff0000u);
  f[2] = __uint_as_float(r.y << 16); f[3] = __uint_as_float(r.y & 0xffff0000u);
}
__device__ __forceinline__ uint2 pack_4(const float* f) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// ROWS rows per block, 8 / ROWS warps on each, all heads in the order query heads, key heads, value heads.
template <int D, int ROWS>
__global__ void __launch_bounds__(kPapThreads, 4)
paged_append_kernel(const PagedAppendArgs a, DeviceStatus* st) {
  constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes, half = D / 2;
  constexpr int kWarps = kPapThreads / 32 / ROWS, kUnits = kWarps * kPerWarp;       // warps of a row, heads that they work on at once
  constexpr int U = kPapAhead;                                  // heads that a group of lanes has in flight
  __shared__ float2 turn_s[ROWS][half];
  const int tid = threadIdx.x, lane = tid & 31, gl = lane % kLanes, rr = (tid >> 5) / kWarps;
  const int unit0 = ((tid >> 5) % kWarps) * kPerWarp + lane / kLanes;
  const long long row0 = (long long)blockIdx.x * ROWS, row = row0 + rr;
  const bool here = row < a.n_rows;
  const int total = here ? a.H + 2 * a.Hkv : 0;
  auto load = [&](int h, uint2& lo, uint2& hi) {
    lo = hi = make_uint2(0u, 0u);
    if (h >= total) return;
    const uint16_t* p = h < a.H ? a.q + (row * a.H + h) * D : h < a.H + a.Hkv ? a.k + (row * a.Hkv + (h - a.H)) * D : a.v + (row * a.Hkv + (h - a.H - a.Hkv)) * D;
    lo = *reinterpret_cast<const uint2*>(p + gl * 4);
    hi = *reinterpret_cast<const uint2*>(p + half + gl * 4);
  };
  griddep_launch();
  const double inv_freq = exp2(-a.log2_theta * (2.0 * (tid % half) / D));       // (depends on no earlier kernel)
  griddep_wait();
  uint2 lo[U], hi[U];
#pragma unroll
  for (int u = 0; u < U; ++u) load(unit0 + u * kUnits, lo[u], hi[u]);
  const int slot = here ? a.slots[row] : -1;
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.f;
  if (a.wq != nullptr) {
    unpack_4(*reinterpret_cast<const uint2*>(a.wq + gl * 4), wq); unpack_4(*reinterpret_cast<const uint2*>(a.wq + half + gl * 4), wq + 4);
    unpack_4(*reinterpret_cast<const uint2*>(a.wk + gl * 4), wk); unpack_4(*reinterpret_cast<const uint2*>(a.wk + half + gl * 4), wk + 4);
  }
  for (int x = tid; x < ROWS * half; x += kPapThreads) {
    const int r = x / half, i = x - r * half;                   // (the same dim every time: the block has a multiple of D / 2 threads)
    if (row0 + r < a.n_rows) {
      double ang = (double)a.positions[row0 + r] * inv_freq;
      ang -= 6.283185307179586 * floor(ang * 0.15915494309189535);
      sincosf((float)ang, &turn_s[r][i].y, &turn_s[r][i].x);
    }
  }
  long long place = -1;                                         // of the row in the store
  if (slot >= 0 && (slot >> a.block_shift) < a.n_blocks)
    place = (long long)(slot >> a.block_shift) * a.block_stride + (slot & ((1 << a.block_shift) - 1)) * a.token_stride;
  else if (slot != -1 && unit0 == 0 && gl == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_APPEND, (int)row, slot);
  __syncthreads();
  float2 cs[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) cs[e] = turn_s[rr][gl * 4 + e];
  for (int u0 = unit0; u0 - unit0 < total; u0 += U * kUnits) {              // (the same trips for a row's lanes: the sums below need whole warps)
    uint2 nlo[U], nhi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) load(u0 + (U + u) * kUnits, nlo[u], nhi[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = u0 + u * kUnits;
      const bool live = h < total, is_q = h < a.H, is_v = h >= a.H + a.Hkv;
      float f[8];
      unpack_4(lo[u], f); unpack_4(hi[u], f + 4);
      if (a.wq != nullptr) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float inv = rsqrtf(ss / (float)D + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = f[e] * inv * (is_q ? wq[e] : wk[e]);
      }
      if (live) {
        float r[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          r[e] = f[e] * cs[e].x - f[4 + e] * cs[e].y;
          r[4 + e] = f[4 + e] * cs[e].x + f[e] * cs[e].y;
        }
        const uint2 rlo = is_v ? lo[u] : pack_4(r), rhi = is_v ? hi[u] : pack_4(r + 4);
        uint16_t* p = is_q ? a.q_out + (row * a.H + h) * D : is_v ? a.store_v + place + (h - a.H - a.Hkv) * a.head_stride : a.store_k + place + (h - a.H) * a.head_stride;
        if (is_q || place >= 0) {
          *reinterpret_cast<uint2*>(p + gl * 4) = rlo;
          *reinterpret_cast<uint2*>(p + half + gl * 4) = rhi;
        }
      }
      lo[u] = nlo[u]; hi[u] = nhi[u];
    }
  }
}

}  // namespace relaxkv

using namespace relaxkv;

extern "C" relaxkv_status relaxkv_qk_norm_rope_append_paged(
    const relaxkv_paged_cache* store, const void* q, const void* k, const void* v, int64_t n_rows, int32_t n_q_heads, int32_t n_kv_heads,
    int32_t head_dim, const void* w_q_norm, const void* w_k_norm, float eps, const int32_t* positions, const int32_t* slots, float theta,
    void* q_out, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_qk_norm_rope_append_paged");
  if (!q || !k || !v || !q_out || !positions || !slots || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out)) return RELAXKV_ERR_INVALID_ARG;
  if (!(theta > 1.f) || !(eps >= 0.f) || (w_q_norm == nullptr) != (w_k_norm == nullptr)) return RELAXKV_ERR_INVALID_ARG;
  if (w_q_norm && (!aligned16(w_q_norm) || !aligned16(w_k_norm))) return RELAXKV_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || n_q_heads < 1 || n_kv_heads < 1 || (head_dim != 64 && head_dim != 128)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  relaxkv_status rc = check_store(store, head_dim);
  if (rc != RELAXKV_OK) return rc;
  if (n_rows == 0) return RELAXKV_OK;
  DeviceStatus* st = status_word();
  const int sms = sm_count_of_current_device();
  if (!st || sms <= 0) return RELAXKV_ERR_CUDA;
  PagedAppendArgs a = {};
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
  a.wq = static_cast<const uint16_t*>(w_q_norm); a.wk = static_cast<const uint16_t*>(w_k_norm);
  a.q_out = static_cast<uint16_t*>(q_out); a.store_k = static_cast<uint16_t*>(store->k); a.store_v = static_cast<uint16_t*>(store->v);
  a.positions = positions; a.slots = slots;
  a.block_stride = store->block_stride; a.token_stride = store->token_stride; a.head_stride = store->head_stride; a.n_rows = n_rows;
  a.n_blocks = store->n_blocks; a.block_shift = 31 - __builtin_clz((unsigned)store->block_size); a.H = n_q_heads; a.Hkv = n_kv_heads;
  a.eps = eps;
  a.log2_theta = log2((double)theta);
  const int n_heads = n_q_heads + 2 * n_kv_heads;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Rows of a block: eight of so few heads that a warp has them all at once (8205 rows of 4 / 1 heads of 64: 5.2 us, 7.8 with four rows); else one
  // while the SMs hold the launch's blocks in two turns or less (40 / 8 heads, 64 rows 4.8 us, 1024 rows 8.5; with four 8.4 and 15.0), four for
  // more (4096 rows 26.8, 8205 rows 49.2; with one 32.5 and 61.3, with two 29.3 and 54.3, with eight 31.0 and 50.3).
  const bool small = n_heads <= kPapAhead * (256 / head_dim);
  const int per = small ? 8 : n_rows <= 8LL * sms ? 1 : 4;
  auto kern = head_dim == 128 ? (per == 8 ? paged_append_kernel<128, 8> : per == 4 ? paged_append_kernel<128, 4> : paged_append_kernel<128, 1>)
                              : (per == 8 ? paged_append_kernel<64, 8> : per == 4 ? paged_append_kernel<64, 4> : paged_append_kernel<64, 1>);
  return cuda_ok(launch_chained(kern, dim3((unsigned)((n_rows + per - 1) / per)), kPapThreads, 0, s, a, st));
}
