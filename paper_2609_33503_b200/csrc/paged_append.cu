// Head norm, rotary embedding and append to the paged store of a step's rows in one pass (relaxkv_qk_norm_rope_append_paged).
//
// Reads Q, K, V once and writes rotated Q and the store's K and V once: bound by HBM for many rows (8205 rows of 40 / 8 heads of 128 with norms, 235 MB,
// 41 us = 5.7 TB/s) and by its latencies (row values, then slot) for few.  D / 8 lanes hold one head, each four dims of its first half and the
// four that they are rotated with, as two 8-byte pieces: the pair meets in one lane, and a warp works on two heads of 128 dims (four of 64) at
// once.  All heads of a row turn by the same angles, so a lane keeps its four (cos, sin) in registers; they are made once per row, one angle per
// thread in double precision, while the first heads are on their way.  With 16-byte pieces, the partner in another lane and the angles read
// from shared memory for every head, this took 101 us, bound by shared memory; then 50, bound by the instructions to issue (76 % of the cycles),
// until products came in pairs, addresses from one base per row and value heads went past the arithmetic.  Two heads per group of lanes are on
// their way while two are worked on, and four blocks share an SM: with one head and six blocks 52 us, with four and three 42.  Values stay in
// fp32 from the load to the one rounding at the store.
#include "continuations.cuh"
#include "sm100_ptx.cuh"

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
  __shared__ __align__(16) float cos_s[ROWS][half], sin_s[ROWS][half], w_s[2][D];      // of the rows; norm weights of query and key heads
  const int tid = threadIdx.x, lane = tid & 31, gl = lane % kLanes, rr = (tid >> 5) / kWarps;
  const int pair0 = ((tid >> 5) % kWarps) * kPerWarp, unit0 = pair0 + lane / kLanes;
  const long long row0 = (long long)blockIdx.x * ROWS, row = row0 + rr;
  const int heads = a.H + a.Hkv, total = row < a.n_rows ? heads + a.Hkv : 0;
  // where this lane's part of head 0 would be, of the three inputs and the three outputs
  const uint16_t *pq = a.q + row * a.H * D + gl * 4, *pk = a.k + (row * a.Hkv - a.H) * D + gl * 4, *pv = a.v + (row * a.Hkv - heads) * D + gl * 4;
  auto load = [&](int h, uint2& lo, uint2& hi) {
    lo = hi = make_uint2(0u, 0u);
    if (h >= total) return;
    const uint16_t* p = (h < a.H ? pq : h < heads ? pk : pv) + h * D;
    lo = *reinterpret_cast<const uint2*>(p);
    hi = *reinterpret_cast<const uint2*>(p + half);
  };
  griddep_launch();
  const double inv_freq = exp2(-a.log2_theta * (2.0 * (tid % half) / D));       // (depends on no earlier kernel)
  griddep_wait();
  uint2 lo[U], hi[U];
#pragma unroll
  for (int u = 0; u < U; ++u) load(unit0 + u * kUnits, lo[u], hi[u]);
  const int slot = total ? a.slots[row] : -1;
  if (a.wq != nullptr && tid < D / 2) {
    const uint2 w = reinterpret_cast<const uint2*>(tid < D / 4 ? a.wq : a.wk)[tid & (D / 4 - 1)];
    unpack_4(w, &w_s[0][tid * 4]);
  }
  for (int x = tid; x < ROWS * half; x += kPapThreads) {
    const int r = x / half, i = x - r * half;                   // (the same dim every time: the block has a multiple of D / 2 threads)
    if (row0 + r < a.n_rows) {
      double ang = (double)a.positions[row0 + r] * inv_freq;
      ang -= 6.283185307179586 * floor(ang * 0.15915494309189535);
      sincosf((float)ang, &sin_s[r][i], &cos_s[r][i]);
    }
  }
  long long place = 0;                                          // of the row in the store
  const bool stored = slot >= 0 && (slot >> a.block_shift) < a.n_blocks;
  if (stored) place = (long long)(slot >> a.block_shift) * a.block_stride + (slot & ((1 << a.block_shift) - 1)) * a.token_stride;
  else if (slot != -1 && unit0 == 0 && gl == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_PAGED_APPEND, (int)row, slot);
  uint16_t *oq = a.q_out + row * a.H * D + gl * 4, *ok = a.store_k + place - a.H * a.head_stride + gl * 4,
           *ov = a.store_v + place - heads * a.head_stride + gl * 4;
  __syncthreads();
  float c[4], s[4], ns[4];
  *reinterpret_cast<float4*>(c) = *reinterpret_cast<const float4*>(&cos_s[rr][gl * 4]);
  *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(&sin_s[rr][gl * 4]);
#pragma unroll
  for (int e = 0; e < 4; ++e) ns[e] = -s[e];
  // (a warp's trips depend on its first head alone: the sums below need whole warps)
  for (int p0 = pair0; p0 < total; p0 += U * kUnits) {
    uint2 nlo[U], nhi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) load(p0 + unit0 - pair0 + (U + u) * kUnits, nlo[u], nhi[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int first = p0 + u * kUnits, h = first + unit0 - pair0;
      if (first < heads) {                                      // (value heads alone: as they are)
        float f[8];
        unpack_4(lo[u], f); unpack_4(hi[u], f + 4);
        if (a.wq != nullptr) {
          float s0, s1;
          ptx::mul2(s0, s1, f[0], f[1], f[0], f[1]);
#pragma unroll
          for (int e = 2; e < 8; e += 2) ptx::fma2(s0, s1, f[e], f[e + 1], f[e], f[e + 1], s0, s1);
          float ss = s0 + s1;
#pragma unroll
          for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          const float inv = rsqrtf(ss * (1.f / D) + a.eps);
          const float* w = w_s[h < a.H ? 0 : 1] + gl * 4;
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float4 wv = *reinterpret_cast<const float4*>(w + hf * half);
            float* x = f + 4 * hf;
            ptx::mul2(x[0], x[1], x[0], x[1], inv, inv);
            ptx::mul2(x[2], x[3], x[2], x[3], inv, inv);
            ptx::mul2(x[0], x[1], x[0], x[1], wv.x, wv.y);
            ptx::mul2(x[2], x[3], x[2], x[3], wv.z, wv.w);
          }
        }
        if (h < heads) {
          float r[8];
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            ptx::mul2(r[e], r[e + 1], f[4 + e], f[5 + e], ns[e], ns[e + 1]);
            ptx::fma2(r[e], r[e + 1], f[e], f[e + 1], c[e], c[e + 1], r[e], r[e + 1]);
            ptx::mul2(r[4 + e], r[5 + e], f[e], f[e + 1], s[e], s[e + 1]);
            ptx::fma2(r[4 + e], r[5 + e], f[4 + e], f[5 + e], c[e], c[e + 1], r[4 + e], r[5 + e]);
          }
          lo[u] = pack_4(r); hi[u] = pack_4(r + 4);
        }
      }
      if (h < total && (h < a.H || stored)) {
        uint16_t* p = h < a.H ? oq + h * D : (h < heads ? ok : ov) + h * a.head_stride;
        *reinterpret_cast<uint2*>(p) = lo[u];
        *reinterpret_cast<uint2*>(p + half) = hi[u];
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
  // Rows of a block: eight of so few heads that a warp has them in four trips (8205 rows of 8 / 2 heads of 128 11.8 us, 14.3 with four rows; of 4 / 1 heads
  // of 64 4.6 and 7.3); else one while the SMs hold the launch's blocks in two turns or less (40 / 8 heads, 64 rows 4.6 us, 1024 rows 7.2; with
  // four 5.9 and 10.4), four for more (2048 rows 12.2, 8205 rows 41.3; with one 15.3 and 51.6, with eight 19.8 and 41.3).
  const bool small = n_heads <= 4 * kPapAhead * (256 / head_dim);
  const int per = small ? 8 : n_rows <= 8LL * sms ? 1 : 4;
  auto kern = head_dim == 128 ? (per == 8 ? paged_append_kernel<128, 8> : per == 4 ? paged_append_kernel<128, 4> : paged_append_kernel<128, 1>)
                              : (per == 8 ? paged_append_kernel<64, 8> : per == 4 ? paged_append_kernel<64, 4> : paged_append_kernel<64, 1>);
  return cuda_ok(launch_chained(kern, dim3((unsigned)((n_rows + per - 1) / per)), kPapThreads, 0, s, a, st));
}
