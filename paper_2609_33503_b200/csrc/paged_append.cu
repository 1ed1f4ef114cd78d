// Head norm, rotary embedding and append to the paged store of a step's rows in one pass (relaxkv_qk_norm_rope_append_paged).
//
// Reads Q, K, V once and writes rotated Q and the store's K and V once: bound by HBM for many rows and by its latencies (row values, then slot) for
// few.  16 lanes hold one head of 128 dims as 16-byte pieces (8 lanes one of 64): a warp works on two (four) heads at once, the rotation partner is
// half of those lanes away.  A block has a few rows; its (cos, sin) table, one angle per thread in double precision, is made while the first
// heads are on their way.  Values stay in fp32 from the load to the one rounding at the store.
#include "continuations.cuh"

namespace relaxkv {

constexpr int kPapThreads = 256;

struct PagedAppendArgs {
  const uint16_t *q, *k, *v, *wq, *wk;
  uint16_t *q_out, *store_k, *store_v;
  const int *positions, *slots;
  long long block_stride, token_stride, head_stride, n_rows;
  int n_blocks, block_shift, H, Hkv;
  float eps;
  double log2_theta;
};

__device__ __forceinline__ void unpack_8(const uint4& r, float* f) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 pack_8(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// ROWS rows per block, heads [blockIdx.y * heads_per_block, + heads_per_block) of each, in the order query heads, key heads, value heads.
template <int D, int ROWS>
__global__ void __launch_bounds__(kPapThreads)
paged_append_kernel(const PagedAppendArgs a, int heads_per_block, DeviceStatus* st) {
  constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes, half = D / 2;
  constexpr int U = 4;                                          // heads a group of lanes has in flight
  __shared__ float2 turn_s[ROWS][half];
  __shared__ long long place_s[ROWS];
  const int tid = threadIdx.x, lane = tid & 31, gl = lane % kLanes, unit0 = (tid >> 5) * kPerWarp + lane / kLanes;
  constexpr int kUnits = (kPapThreads / 32) * kPerWarp;         // heads the block works on at once
  const long long row0 = (long long)blockIdx.x * ROWS;
  const int n_heads = a.H + 2 * a.Hkv, h0 = blockIdx.y * heads_per_block, n_here = min(heads_per_block, n_heads - h0);
  const int rows_here = (int)min((long long)ROWS, a.n_rows - row0), total = rows_here * n_here;
  const bool low = gl < kLanes / 2;
  auto load = [&](int u) -> uint4 {
    if (u >= total) return make_uint4(0, 0, 0, 0);
    const int rr = u / n_here, h = h0 + u - rr * n_here;
    const long long row = row0 + rr;
    const uint16_t* p = h < a.H ? a.q + (row * a.H + h) * D : h < a.H + a.Hkv ? a.k + (row * a.Hkv + (h - a.H)) * D : a.v + (row * a.Hkv + (h - a.H - a.Hkv)) * D;
    return *reinterpret_cast<const uint4*>(p + gl * 8);
  };
  griddep_launch();
  griddep_wait();
  uint4 raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) raw[u] = load(unit0 + u * kUnits);
  for (int x = tid; x < ROWS * half; x += kPapThreads) {
    const int rr = x / half, i = x - rr * half;
    if (rr < rows_here) {
      const double inv_freq = exp2(-a.log2_theta * (2.0 * i / D));
      double ang = (double)a.positions[row0 + rr] * inv_freq;
      ang -= 6.283185307179586 * floor(ang * 0.15915494309189535);
      sincosf((float)ang, &turn_s[rr][i].y, &turn_s[rr][i].x);
    }
  }
  if (tid < rows_here) {
    const int slot = a.slots[row0 + tid];
    long long place = -1;
    if (slot >= 0 && (slot >> a.block_shift) < a.n_blocks)
      place = (long long)(slot >> a.block_shift) * a.block_stride + (slot & ((1 << a.block_shift) - 1)) * a.token_stride;
    else if (slot != -1 && blockIdx.y == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_APPEND, (int)(row0 + tid), slot);
    place_s[tid] = place;
  }
  __syncthreads();
  for (int u0 = unit0; u0 - unit0 < total; u0 += U * kUnits) {              // (the same trips for all lanes: the sums below need whole warps)
    uint4 next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = load(u0 + (U + u) * kUnits);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = u0 + u * kUnits;
      const bool live = x < total;
      const int rr = live ? x / n_here : 0, h = live ? h0 + x - rr * n_here : 0;
      const bool is_v = h >= a.H + a.Hkv;
      float f[8];
      unpack_8(raw[u], f);
      if (a.wq != nullptr) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(f[e], f[e], ss);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float inv = rsqrtf(ss / (float)D + a.eps);
        if (live && !is_v) {
          float w[8];
          unpack_8(*reinterpret_cast<const uint4*>((h < a.H ? a.wq : a.wk) + gl * 8), w);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = f[e] * inv * w[e];
        }
      }
      float r[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float other = __shfl_xor_sync(0xffffffffu, f[e], kLanes / 2);
        const float2 cs = turn_s[rr][(gl % (kLanes / 2)) * 8 + e];
        r[e] = low ? f[e] * cs.x - other * cs.y : f[e] * cs.x + other * cs.y;
      }
      if (live) {
        const long long place = place_s[rr];
        if (h < a.H) *reinterpret_cast<uint4*>(a.q_out + ((row0 + rr) * a.H + h) * D + gl * 8) = pack_8(r);
        else if (place >= 0) {
          if (is_v) *reinterpret_cast<uint4*>(a.store_v + place + (h - a.H - a.Hkv) * a.head_stride + gl * 8) = raw[u];
          else *reinterpret_cast<uint4*>(a.store_k + place + (h - a.H) * a.head_stride + gl * 8) = pack_8(r);
        }
      }
      raw[u] = next[u];
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
  if (!st) return RELAXKV_ERR_CUDA;
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
  if (n_rows >= 1024) {                         // four rows per block: every thread makes one angle or two
    const dim3 grid((unsigned)((n_rows + 3) / 4), 1);
    auto kern = head_dim == 128 ? paged_append_kernel<128, 4> : paged_append_kernel<64, 4>;
    return cuda_ok(launch_chained(kern, grid, kPapThreads, 0, s, a, n_heads, st));
  }
  const int per = head_dim == 128 ? 16 : 32;    // one head per group of lanes
  const dim3 grid((unsigned)n_rows, (unsigned)((n_heads + per - 1) / per));
  auto kern = head_dim == 128 ? paged_append_kernel<128, 1> : paged_append_kernel<64, 1>;
  return cuda_ok(launch_chained(kern, grid, kPapThreads, 0, s, a, per, st));
}
