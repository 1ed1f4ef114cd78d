// Rotary embeddings of every form (relaxkv_qk_norm_rotate), rows into the 8-bit store (relaxkv_append_quantized) and back
// (relaxkv_read_quantized).
//
// All three read and write every element once and are bound by HBM for many rows, by their latencies (row values, then slot or
// angle) for few.  D / 8 lanes hold a head, eight dims each, chosen so that a pair always meets in one lane: dims 8 i .. 8 i + 7
// where pairs are neighbours or nothing turns; where pair i is (i, i + part / 2), dims 4 i .. and part / 2 + 4 i .. of the part
// that turns, and the dims behind it eight at a time.  Lane i has the pairs 4 i .. 4 i + 3 either way.  All heads of a row turn by
// the same angles, which are made once per row, one per thread: the turns p freq / 2 pi are rounded to their remainder in fp64 (a
// float of position 100000 would be off by 2^-8 radians), sine and cosine of that in fp32, with what its own rounding cuts off
// (which moved a third of the keys that land on the other side of a rounding to 8 bits than the formula's: 18 of 4 million e4m3
// values for 32).  Everything else stays in fp32 until the one rounding at the end.  The scale of 8 bits is a power of two: the
// division by it is exact, values of two eighths of bf16's bits stay exact when read back, and the bytes do not depend on the order
// of anything.
//
// Measured (L2 flushed): 8205 rows of 40 / 8 heads with norms, half the head turned, 40 us (5.0 TB/s of bytes that have to move);
// 16 K rows of 8 heads written as e4m3 and read back 34.5 us (by themselves 19 and 18); 32 K rows read and turned 40 (5.1 TB/s); 64
// rows of 32 / 8 heads turned 5.2, written and read back 9.6.  Many rows with norm and rotation issue in 78 % of the schedulers'
// cycles: some 160 instructions for eight elements with their addresses.  Sixteen elements to a lane took longer (50.7 us; 45.9
// read), fewer heads being in flight.
#include "quantized_cache.cuh"
#include "sm100_ptx.cuh"
#include <cmath>

namespace relaxkv {

constexpr int kTurnThreads = 256, kTurnAhead = 2;

enum TurnStore { STORE_BF16 = 0, STORE_INT8 = 1, STORE_E4M3 = 2 };

struct TurnArgs {
  const uint16_t *q, *k, *v, *wq, *wk;
  uint16_t *q_out, *k_out, *v_out;
  uint8_t *store_k, *store_v;
  int8_t *exp_k, *exp_v;
  const int *positions, *slots;
  const double* freq;
  long long q_token, k_token;                            // strides of the bf16 rows
  long long block_stride, token_stride;                  // of the store
  int q_head, k_head, head_stride;                       // from head to head
  long long n_rows;
  int n_blocks, block_shift, H, Hkv;
  int part;                                              // dims that turn, 0: none
  float eps, amplitude;
};

__device__ __forceinline__ void unpack_8(const uint2& lo, const uint2& hi, float* f) {
  const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint2 pack_bf16(const float* f) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
  return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// First dims of a lane's two runs of four.
template <bool HALF>
__device__ __forceinline__ void lane_dims(int gl, int part, int* lo, int* hi) {
  const bool turned = HALF && gl < part / 8;
  *lo = turned ? 4 * gl : 8 * gl;
  *hi = turned ? part / 2 + 4 * gl : 8 * gl + 4;
}

// Eight elements by the four angles (cosine c, sine s, -s) of their pairs: element i and i + 4, or 2 i and 2 i + 1.
template <bool HALF>
__device__ __forceinline__ void turn_8(float* f, const float* c, const float* s, const float* ns) {
  if constexpr (HALF) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      float x0, x1, y0, y1;
      ptx::mul2(x0, x1, f[i + 4], f[i + 5], ns[i], ns[i + 1]);
      ptx::fma2(x0, x1, f[i], f[i + 1], c[i], c[i + 1], x0, x1);
      ptx::mul2(y0, y1, f[i], f[i + 1], s[i], s[i + 1]);
      ptx::fma2(y0, y1, f[i + 4], f[i + 5], c[i], c[i + 1], y0, y1);
      f[i] = x0; f[i + 1] = x1; f[i + 4] = y0; f[i + 5] = y1;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = f[2 * i], b = f[2 * i + 1];
      f[2 * i] = fmaf(a, c[i], b * ns[i]);
      f[2 * i + 1] = fmaf(b, c[i], a * s[i]);
    }
  }
}

__device__ __forceinline__ float largest_3(float a, float b, float c) {        // of absolute values; NaN where one is
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
  return d;
}

// Cosines and sines of the block's rows, [ROWS][part / 2], one per thread at a time.
template <int ROWS, int HALF_DIMS>
__device__ __forceinline__ void make_angles(const int* positions, const double* freq, int pairs, float amplitude, long long row0, long long n_rows,
                                            float (*cos_s)[HALF_DIMS], float (*sin_s)[HALF_DIMS]) {
  for (int x = threadIdx.x; x < ROWS * pairs; x += kTurnThreads) {
    const int r = x / pairs, i = x - r * pairs;
    if (row0 + r >= n_rows) break;
    double turns = (double)positions[row0 + r] * (freq[i] * 0.15915494309189535);
    turns -= rint(turns);
    const float near = (float)turns, rest = (float)(turns - near) * 6.28318531f;       // (what the rounding cuts off, up to 2^-23 radians)
    float s, c;
    sincospif(2.f * near, &s, &c);
    cos_s[r][i] = amplitude * fmaf(-s, rest, c);
    sin_s[r][i] = amplitude * fmaf(c, rest, s);
  }
}

// Exponent of a token and head from the largest of its elements' bits without their signs (an infinity or NaN is larger than every number).
template <int STORE>
__device__ __forceinline__ int store_exponent(uint32_t largest) {
  constexpr uint32_t kMantissa = STORE == STORE_INT8 ? 0x7e0000u : 0x600000u;         // of 127 = 1.984375 * 2^6 and 448 = 1.75 * 2^8
  constexpr int kTop = STORE == STORE_INT8 ? 6 : 8;
  if (largest >= 0x7f800000u) return kExpNone;
  const int e = (int)(largest >> 23) - 127 - kTop + ((largest & 0x7fffffu) > kMantissa ? 1 : 0);
  return max(e, kExpLeast);
}

// Four numbers as bytes of the store, inv = 2^-exponent.
template <int STORE>
__device__ __forceinline__ uint32_t store_bytes(const float* f, float inv) {
  if constexpr (STORE == STORE_INT8) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(fmaf(f[i], inv, 12582912.f));  // 1.5 * 2^23: the whole number stands in the low bits
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  } else {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(f[1] * inv), "f"(f[0] * inv));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(f[3] * inv), "f"(f[2] * inv));
    return (uint32_t)lo | ((uint32_t)hi << 16);
  }
}

// ROWS rows per block, 8 / ROWS warps on each, all heads in the order query heads, key heads, value heads (these only where there is a store).
template <int D, bool HALF, int STORE, int ROWS>
__global__ void __launch_bounds__(kTurnThreads, 4)
turn_rows_kernel(const TurnArgs a, DeviceStatus* st) {
  constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes, kHalf = D / 2;
  constexpr int kWarps = kTurnThreads / 32 / ROWS, kUnits = kWarps * kPerWarp;      // warps of a row, heads that they work on at once
  constexpr int U = kTurnAhead;                                // heads that a group of lanes has in flight
  __shared__ __align__(16) float cos_s[ROWS][kHalf], sin_s[ROWS][kHalf], w_s[2][D];
  const int tid = threadIdx.x, lane = tid & 31, gl = lane % kLanes, rr = (tid >> 5) / kWarps;
  const int pair0 = ((tid >> 5) % kWarps) * kPerWarp, unit0 = pair0 + lane / kLanes;
  const long long row0 = (long long)blockIdx.x * ROWS, row = row0 + rr;
  const int heads = a.H + a.Hkv, total = row < a.n_rows ? heads + (STORE != STORE_BF16 ? a.Hkv : 0) : 0;
  int dlo, dhi;
  lane_dims<HALF>(gl, a.part, &dlo, &dhi);
  const bool turned = gl < a.part / 8;
  // where this lane's part of head 0 would be, of the inputs and outputs, if all heads stood there one behind the other
  const long long q_at = row * a.q_token + dlo, k_at = row * a.k_token - (long long)a.H * a.k_head + dlo;
  const uint16_t *pq = a.q + q_at, *pk = a.k + k_at, *pv = a.v + k_at - (long long)a.Hkv * a.k_head;
  const int dd = dhi - dlo;
  auto load = [&](int h, uint2& lo, uint2& hi) {
    lo = hi = make_uint2(0u, 0u);
    if (h >= total) return;
    const bool of_q = h < a.H;
    const uint16_t* p = (of_q ? pq : h < heads ? pk : pv) + (long long)h * (of_q ? a.q_head : a.k_head);
    if constexpr (HALF) {
      lo = *reinterpret_cast<const uint2*>(p);
      hi = *reinterpret_cast<const uint2*>(p + dd);
    } else {
      const uint4 w = *reinterpret_cast<const uint4*>(p);
      lo = make_uint2(w.x, w.y); hi = make_uint2(w.z, w.w);
    }
  };
  griddep_launch();
  griddep_wait();
  uint2 lo[U], hi[U];
#pragma unroll
  for (int u = 0; u < U; ++u) load(unit0 + u * kUnits, lo[u], hi[u]);
  const int slot = STORE != STORE_BF16 && total ? a.slots[row] : -1;
  if (a.wq != nullptr)
    for (int x = tid; x < 2 * D; x += kTurnThreads) w_s[x / D][x % D] = bf16_bits_to_float((x < D ? a.wq : a.wk)[x % D]);
  if (a.part > 0) make_angles<ROWS>(a.positions, a.freq, a.part / 2, a.amplitude, row0, a.n_rows, cos_s, sin_s);
  long long at = 0, exp_at = 0;                                // of the row in the store
  const bool stored = slot >= 0 && (slot >> a.block_shift) < a.n_blocks;
  if (stored) {
    const int block = slot >> a.block_shift, token = slot & ((1 << a.block_shift) - 1);
    at = block * a.block_stride + token * a.token_stride;
    exp_at = (((long long)block * a.Hkv) << a.block_shift) + token;
  } else if (STORE != STORE_BF16 && slot != -1 && unit0 == 0 && gl == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ROWS, (int)row, slot);
  uint16_t *oq = a.q_out + q_at, *ok = a.k_out + k_at;
  uint8_t *sk = a.store_k + at - (long long)a.H * a.head_stride + dlo, *sv = a.store_v + at - (long long)heads * a.head_stride + dlo;
  __syncthreads();
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f}, ns[4];
  if (turned) {
    *reinterpret_cast<float4*>(c) = *reinterpret_cast<const float4*>(&cos_s[rr][gl * 4]);
    *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(&sin_s[rr][gl * 4]);
  }
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
      float f[8];
      unpack_8(lo[u], hi[u], f);
      if (first < heads && a.wq != nullptr) {
        float s0, s1;
        ptx::mul2(s0, s1, f[0], f[1], f[0], f[1]);
#pragma unroll
        for (int e = 2; e < 8; e += 2) ptx::fma2(s0, s1, f[e], f[e + 1], f[e], f[e + 1], s0, s1);
        float ss = s0 + s1;
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        if (h < heads) {
          const float inv = rsqrtf(ss * (1.f / D) + a.eps);
          const float* w = w_s[h < a.H ? 0 : 1];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float4 wv = *reinterpret_cast<const float4*>(w + (hf ? dhi : dlo));
            float* x = f + 4 * hf;
            ptx::mul2(x[0], x[1], x[0], x[1], inv, inv);
            ptx::mul2(x[2], x[3], x[2], x[3], inv, inv);
            ptx::mul2(x[0], x[1], x[0], x[1], wv.x, wv.y);
            ptx::mul2(x[2], x[3], x[2], x[3], wv.z, wv.w);
          }
        }
      }
      if (turned && h < heads) turn_8<HALF>(f, c, s, ns);
      if (STORE == STORE_BF16 || first < a.H) {
        if (h < total && (STORE == STORE_BF16 || h < a.H)) {
          uint16_t* p = (STORE != STORE_BF16 || h < a.H ? oq : ok) + (long long)h * (STORE != STORE_BF16 || h < a.H ? a.q_head : a.k_head);
          const bool changed = turned || a.wq != nullptr;        // (what stays keeps every bit, those of a NaN too)
          const uint2 r0 = changed ? pack_bf16(f) : lo[u], r1 = changed ? pack_bf16(f + 4) : hi[u];
          if constexpr (HALF) {
            *reinterpret_cast<uint2*>(p) = r0;
            *reinterpret_cast<uint2*>(p + dd) = r1;
          } else *reinterpret_cast<uint4*>(p) = make_uint4(r0.x, r0.y, r1.x, r1.y);
        }
      }
      if (STORE != STORE_BF16 && first + kPerWarp > a.H) {     // some of this warp's heads go to the store
        const float t0 = largest_3(fabsf(f[0]), f[1], f[2]), t1 = largest_3(fabsf(f[3]), f[4], f[5]);
        uint32_t top = __float_as_uint(largest_3(largest_3(t0, f[6], f[7]), t1, t1));       // (the order of bits is that of numbers, infinity, NaN)
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (stored && h >= a.H && h < total) {
          const int e = store_exponent<STORE>(top);
          const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
          uint32_t b0 = 0, b1 = 0;
          if (e != kExpNone) { b0 = store_bytes<STORE>(f, inv); b1 = store_bytes<STORE>(f + 4, inv); }
          uint8_t* p = (h < heads ? sk : sv) + (long long)h * a.head_stride;
          if constexpr (HALF) {
            *reinterpret_cast<uint32_t*>(p) = b0;
            *reinterpret_cast<uint32_t*>(p + dd) = b1;
          } else *reinterpret_cast<uint2*>(p) = make_uint2(b0, b1);
          if (gl == 0) (h < heads ? a.exp_k : a.exp_v)[exp_at + ((h < heads ? h - a.H : h - heads) << a.block_shift)] = (int8_t)e;
        }
      }
      lo[u] = nlo[u]; hi[u] = nhi[u];
    }
  }
}

// Eight values of the store by their scale.
template <int TYPE>
__device__ __forceinline__ void scaled_8(const uint32_t* w, float scale, float* f) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (TYPE == RELAXKV_INT8) {                      // 2^23 + 128 + value, less 2^23 + 128: exact, and only then the scale, which is up to 2^127
      const uint32_t b = w[i] ^ 0x80808080u;
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        float* x = f + 4 * i + j;
        x[0] = __uint_as_float(__byte_perm(b, 0x4b000000u, 0x7550 | j));
        x[1] = __uint_as_float(__byte_perm(b, 0x4b000000u, 0x7550 | (j + 1)));
        ptx::add2(x[0], x[1], -8388736.f, -8388736.f);
        ptx::mul2(x[0], x[1], x[0], x[1], scale, scale);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t p = e4m3_to_half2(w[i], j);
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&p));
        f[4 * i + 2 * j] = v.x * scale; f[4 * i + 2 * j + 1] = v.y * scale;
      }
    }
  }
}

// Rows of the store as bf16, the keys turned.  A key head and its value head lie alike, in the store and in the rows: one address for both.
template <int D, bool HALF, int TYPE, int ROWS>
__global__ void __launch_bounds__(kTurnThreads, 4)
read_rows_kernel(const TurnArgs a, DeviceStatus* st) {
  constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes, kHalf = D / 2;
  constexpr int kWarps = kTurnThreads / 32 / ROWS, kUnits = kWarps * kPerWarp, U = kTurnAhead;
  __shared__ __align__(16) float cos_s[ROWS][kHalf], sin_s[ROWS][kHalf];
  const int tid = threadIdx.x, lane = tid & 31, gl = lane % kLanes, rr = (tid >> 5) / kWarps;
  const int unit0 = ((tid >> 5) % kWarps) * kPerWarp + lane / kLanes;
  const long long row0 = (long long)blockIdx.x * ROWS, row = row0 + rr;
  int dlo, dhi;
  lane_dims<HALF>(gl, a.part, &dlo, &dhi);
  const bool turned = gl < a.part / 8;
  griddep_launch();
  griddep_wait();
  const int slot = row < a.n_rows ? a.slots[row] : -1;
  const bool stored = slot >= 0 && (slot >> a.block_shift) < a.n_blocks;
  const int heads = stored ? a.Hkv : 0;
  const int block = stored ? slot >> a.block_shift : 0, token = stored ? slot & ((1 << a.block_shift) - 1) : 0;
  const long long at = block * a.block_stride + token * a.token_stride + dlo, exp_at = (((long long)block * a.Hkv) << a.block_shift) + token;
  if (!stored && slot != -1 && unit0 == 0 && gl == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ROWS, (int)row, slot);
  const int dd = dhi - dlo;
  uint32_t w[U][2][2];
  int e[U][2];
  auto load = [&](int u, int h) {
    if (h >= heads) return;
    const long long off = at + (long long)h * a.head_stride, eo = exp_at + (h << a.block_shift);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t* p = (t == 0 ? a.store_k : a.store_v) + off;
      if constexpr (HALF) {
        w[u][t][0] = *reinterpret_cast<const uint32_t*>(p);
        w[u][t][1] = *reinterpret_cast<const uint32_t*>(p + dd);
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        w[u][t][0] = x.x; w[u][t][1] = x.y;
      }
      e[u][t] = (t == 0 ? a.exp_k : a.exp_v)[eo];
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u) load(u, unit0 + u * kUnits);
  make_angles<ROWS>(a.positions, a.freq, a.part / 2, a.amplitude, row0, a.n_rows, cos_s, sin_s);
  __syncthreads();
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f}, ns[4];
  if (turned) {
    *reinterpret_cast<float4*>(c) = *reinterpret_cast<const float4*>(&cos_s[rr][gl * 4]);
    *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(&sin_s[rr][gl * 4]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) ns[i] = -s[i];
  uint16_t *ok = a.k_out + row * a.k_token + dlo, *ov = a.v_out + row * a.k_token + dlo;
  for (int h0 = unit0; h0 < heads; h0 += U * kUnits) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * kUnits;
      if (h >= heads) break;
      const long long off = (long long)h * a.k_head;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float f[8];
        scaled_8<TYPE>(w[u][t], exp_scale(e[u][t]), f);
        if (t == 0 && turned) turn_8<HALF>(f, c, s, ns);
        uint16_t* out = (t == 0 ? ok : ov) + off;
        const uint2 r0 = pack_bf16(f), r1 = pack_bf16(f + 4);
        if constexpr (HALF) {
          *reinterpret_cast<uint2*>(out) = r0;
          *reinterpret_cast<uint2*>(out + dd) = r1;
        } else *reinterpret_cast<uint4*>(out) = make_uint4(r0.x, r0.y, r1.x, r1.y);
      }
      load(u, h + U * kUnits);
    }
  }
}

// Rows that go to the store, or come from it, as they are.  A warp has a row's key heads and value heads, which lie alike, side by side: one address, one exchange of the largest
// elements (16 bits each) for both.  (As a case of the kernels above, 170 instructions for eight elements of two heads in place of 50; 16 K rows of 8 heads to
// e4m3 and back 45 us, so 34.5.  Two or four heads ahead of the one at work 35.4.)
template <int D, int STORE, int ROWS>
__global__ void __launch_bounds__(kTurnThreads)
store_plain_rows_kernel(const TurnArgs a, DeviceStatus* st) {
  constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes, kWarps = kTurnThreads / 32 / ROWS, kUnits = kWarps * kPerWarp;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane % kLanes, h0 = (warp % kWarps) * kPerWarp;
  const long long row = (long long)blockIdx.x * ROWS + warp / kWarps;
  griddep_launch();
  griddep_wait();
  if (row >= a.n_rows) return;
  const int slot = a.slots[row];
  const uint16_t *pk = a.k + row * a.k_token + gl * 8, *pv = a.v + row * a.k_token + gl * 8;
  const bool stored = slot >= 0 && (slot >> a.block_shift) < a.n_blocks;
  if (!stored && slot != -1 && h0 == 0 && lane == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ROWS, (int)row, slot);
  const int block = slot >> a.block_shift, token = slot & ((1 << a.block_shift) - 1);
  const long long at = block * a.block_stride + token * a.token_stride + gl * 8, exp_at = (((long long)block * a.Hkv) << a.block_shift) + token;
  for (int h1 = h0; h1 < a.Hkv; h1 += kUnits) {              // (the same for all lanes)
    const int h = h1 + lane / kLanes;
    uint4 x[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
    if (h < a.Hkv) {                                         // (read for the last time: what L2 keeps is the store)
      x[0] = __ldcs(reinterpret_cast<const uint4*>(pk + (long long)h * a.k_head));
      x[1] = __ldcs(reinterpret_cast<const uint4*>(pv + (long long)h * a.k_head));
    }
    uint32_t top[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      constexpr uint32_t kNoSign = 0x7fff7fffu;
      top[t] = __vmaxu2(__vmaxu2(x[t].x & kNoSign, x[t].y & kNoSign), __vmaxu2(x[t].z & kNoSign, x[t].w & kNoSign));
    }
    uint32_t both = __vmaxu2(__byte_perm(top[0], top[1], 0x5410), __byte_perm(top[0], top[1], 0x7632));      // keys below, values above
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, o));
    if (!stored || h >= a.Hkv) continue;
    const int e[2] = {store_exponent<STORE>(both << 16), store_exponent<STORE>(both & 0xffff0000u)};
    const long long off = at + (long long)h * a.head_stride;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float f[8];
      unpack_8(make_uint2(x[t].x, x[t].y), make_uint2(x[t].z, x[t].w), f);
      const float inv = __uint_as_float((uint32_t)(127 - e[t]) << 23);
      uint2 b = make_uint2(store_bytes<STORE>(f, inv), store_bytes<STORE>(f + 4, inv));
      if (e[t] == kExpNone) b = make_uint2(0u, 0u);
      *reinterpret_cast<uint2*>((t == 0 ? a.store_k : a.store_v) + off) = b;
    }
    if (gl < 2) (gl == 0 ? a.exp_k : a.exp_v)[exp_at + (h << a.block_shift)] = (int8_t)(gl == 0 ? e[0] : e[1]);
  }
}

template <int D, int TYPE, int ROWS>
__global__ void __launch_bounds__(kTurnThreads)
read_plain_rows_kernel(const TurnArgs a, DeviceStatus* st) {
  constexpr int kLanes = D / 8, kPerWarp = 32 / kLanes, kWarps = kTurnThreads / 32 / ROWS, kUnits = kWarps * kPerWarp, U = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane % kLanes, h0 = (warp % kWarps) * kPerWarp;
  const long long row = (long long)blockIdx.x * ROWS + warp / kWarps;
  griddep_launch();
  griddep_wait();
  if (row >= a.n_rows) return;
  const int slot = a.slots[row];
  if (slot < 0 || (slot >> a.block_shift) >= a.n_blocks) {
    if (slot != -1 && h0 == 0 && lane == 0) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ROWS, (int)row, slot);
    return;
  }
  const int block = slot >> a.block_shift, token = slot & ((1 << a.block_shift) - 1);
  const long long at = block * a.block_stride + token * a.token_stride + gl * 8, exp_at = (((long long)block * a.Hkv) << a.block_shift) + token;
  uint16_t *ok = a.k_out + row * a.k_token + gl * 8, *ov = a.v_out + row * a.k_token + gl * 8;
  for (int h1 = h0 + lane / kLanes; h1 < a.Hkv; h1 += U * kUnits) {
    uint2 w[U][2];
    int e[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h1 + u * kUnits;
      if (h >= a.Hkv) break;
      const long long off = at + (long long)h * a.head_stride, eo = exp_at + (h << a.block_shift);
      w[u][0] = *reinterpret_cast<const uint2*>(a.store_k + off);
      w[u][1] = *reinterpret_cast<const uint2*>(a.store_v + off);
      e[u][0] = a.exp_k[eo];
      e[u][1] = a.exp_v[eo];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h1 + u * kUnits;
      if (h >= a.Hkv) break;
      const long long off = (long long)h * a.k_head;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t x[2] = {w[u][t].x, w[u][t].y};
        float f[8];
        scaled_8<TYPE>(x, exp_scale(e[u][t]), f);
        const uint2 r0 = pack_bf16(f), r1 = pack_bf16(f + 4);
        *reinterpret_cast<uint4*>((t == 0 ? ok : ov) + off) = make_uint4(r0.x, r0.y, r1.x, r1.y);
      }
    }
  }
}

template <int D, bool HALF, int STORE>
static cudaError_t launch_turn(const TurnArgs& a, int per, DeviceStatus* st, cudaStream_t stream) {
  auto kern = per == 8 ? turn_rows_kernel<D, HALF, STORE, 8> : per == 4 ? turn_rows_kernel<D, HALF, STORE, 4> : turn_rows_kernel<D, HALF, STORE, 1>;
  return launch_chained(kern, dim3((unsigned)((a.n_rows + per - 1) / per)), kTurnThreads, 0, stream, a, st);
}
template <int STORE>
static cudaError_t launch_turn_d(int D, bool half, const TurnArgs& a, int per, DeviceStatus* st, cudaStream_t stream) {
  if (D == 128) return half ? launch_turn<128, true, STORE>(a, per, st, stream) : launch_turn<128, false, STORE>(a, per, st, stream);
  return half ? launch_turn<64, true, STORE>(a, per, st, stream) : launch_turn<64, false, STORE>(a, per, st, stream);
}
template <int D, bool HALF, int TYPE>
static cudaError_t launch_read(const TurnArgs& a, int per, DeviceStatus* st, cudaStream_t stream) {
  auto kern = per == 8 ? read_rows_kernel<D, HALF, TYPE, 8> : per == 4 ? read_rows_kernel<D, HALF, TYPE, 4> : read_rows_kernel<D, HALF, TYPE, 1>;
  return launch_chained(kern, dim3((unsigned)((a.n_rows + per - 1) / per)), kTurnThreads, 0, stream, a, st);
}

template <int D, int STORE>
static cudaError_t launch_store_plain(const TurnArgs& a, int per, DeviceStatus* st, cudaStream_t stream) {
  auto kern = per == 8 ? store_plain_rows_kernel<D, STORE, 8> : per == 4 ? store_plain_rows_kernel<D, STORE, 4> : store_plain_rows_kernel<D, STORE, 1>;
  return launch_chained(kern, dim3((unsigned)((a.n_rows + per - 1) / per)), kTurnThreads, 0, stream, a, st);
}
template <int D, int TYPE>
static cudaError_t launch_read_plain(const TurnArgs& a, int per, DeviceStatus* st, cudaStream_t stream) {
  auto kern = per == 8 ? read_plain_rows_kernel<D, TYPE, 8> : per == 4 ? read_plain_rows_kernel<D, TYPE, 4> : read_plain_rows_kernel<D, TYPE, 1>;
  return launch_chained(kern, dim3((unsigned)((a.n_rows + per - 1) / per)), kTurnThreads, 0, stream, a, st);
}

static relaxkv_status check_rotary(const relaxkv_rotary* r, const int32_t* positions, int head_dim) {
  if (!r) return RELAXKV_OK;
  if (!r->freq || (reinterpret_cast<uintptr_t>(r->freq) & 7u) || !positions) return RELAXKV_ERR_INVALID_ARG;
  if (r->dims < 0 || r->dims % 8 || r->dims > head_dim || (r->interleaved != 0 && r->interleaved != 1)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (!(r->amplitude > 0.f) || !std::isfinite(r->amplitude)) return RELAXKV_ERR_INVALID_ARG;
  return RELAXKV_OK;
}
static bool bf16_rows_ok(const void* p, const void* out, int64_t token, int64_t head, int head_dim) {
  return p && out && aligned16(p) && aligned16(out) && token >= head_dim && head >= head_dim && head <= 0x7fffffff && token % 8 == 0 && head % 8 == 0;
}
static void set_rotary(TurnArgs& a, const relaxkv_rotary* r, const int32_t* positions) {
  if (!r) return;
  a.freq = r->freq; a.part = r->dims; a.amplitude = r->amplitude; a.positions = positions;
}
static void set_store(TurnArgs& a, const relaxkv_quantized_cache* c) {
  a.store_k = static_cast<uint8_t*>(c->k); a.store_v = static_cast<uint8_t*>(c->v); a.exp_k = c->k_exp; a.exp_v = c->v_exp;
  a.block_stride = c->block_stride; a.token_stride = c->token_stride; a.head_stride = (int)c->head_stride;
  a.n_blocks = c->n_blocks; a.block_shift = 31 - __builtin_clz((unsigned)c->block_size);
}
// Rows of a block: eight of so few heads that a warp has them in four trips, else one while the SMs hold the launch's blocks in two turns or less, four for more.
static int rows_per_block(int64_t n_rows, int heads, int head_dim, int sms) {
  return heads <= 4 * kTurnAhead * (256 / head_dim) ? 8 : n_rows <= 8LL * sms ? 1 : 4;
}

}  // namespace relaxkv

using namespace relaxkv;

extern "C" relaxkv_status relaxkv_rotary_frequencies(int32_t dims, double theta, int32_t scaling, double factor, int32_t original_len, double low,
                                                     double high, double* h_freq_out, float* h_amplitude_out) {
  if (!h_freq_out || !h_amplitude_out || !(theta > 1.0) || !std::isfinite(theta)) return RELAXKV_ERR_INVALID_ARG;
  if (dims < 8 || dims % 8) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (scaling < RELAXKV_SCALE_NONE || scaling > RELAXKV_SCALE_RAMP) return RELAXKV_ERR_INVALID_ARG;
  if (scaling != RELAXKV_SCALE_NONE && (!(factor >= 1.0) || !std::isfinite(factor))) return RELAXKV_ERR_INVALID_ARG;
  if (scaling >= RELAXKV_SCALE_BANDS && (original_len < 1 || !(low > 0.0) || !(high > low) || !std::isfinite(high))) return RELAXKV_ERR_INVALID_ARG;
  constexpr double kTwoPi = 6.283185307179586;
  double from = 0.0, to = 0.0;
  if (scaling == RELAXKV_SCALE_RAMP) {                      // pair (as dim / 2) that makes t turns in original_len positions: theta^(-2 i / dims) original_len = 2 pi t
    auto pair_of = [&](double t) { return dims * std::log(original_len / (kTwoPi * t)) / (2.0 * std::log(theta)); };
    from = std::fmax(std::floor(pair_of(high)), 0.0);
    to = std::fmin(std::ceil(pair_of(low)), dims - 1.0);
  }
  for (int i = 0; i < dims / 2; ++i) {
    const double f = std::pow(theta, -2.0 * i / dims);
    double keep = 1.0;                                      // share of the frequency that is not scaled
    if (scaling == RELAXKV_SCALE_LINEAR) keep = 0.0;
    if (scaling == RELAXKV_SCALE_BANDS) keep = (original_len * f / kTwoPi - low) / (high - low);
    if (scaling == RELAXKV_SCALE_RAMP) keep = 1.0 - (i - from) / std::fmax(to - from, 1e-3);
    keep = std::fmin(1.0, std::fmax(0.0, keep));
    h_freq_out[i] = scaling == RELAXKV_SCALE_NONE ? f : f * (keep + (1.0 - keep) / factor);
  }
  *h_amplitude_out = scaling == RELAXKV_SCALE_RAMP ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return RELAXKV_OK;
}

extern "C" relaxkv_status relaxkv_qk_norm_rotate(
    const void* q, void* q_out, int64_t q_token_stride, int64_t q_head_stride, const void* k, void* k_out, int64_t k_token_stride, int64_t k_head_stride,
    int64_t n_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* w_q_norm, const void* w_k_norm, float eps, const int32_t* positions,
    const relaxkv_rotary* rotary, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_qk_norm_rotate");
  if ((!q && !k) || (q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || !rotary) return RELAXKV_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || (q && n_q_heads < 1) || (k && n_kv_heads < 1) || (head_dim != 64 && head_dim != 128)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if ((q && !bf16_rows_ok(q, q_out, q_token_stride, q_head_stride, head_dim)) || (k && !bf16_rows_ok(k, k_out, k_token_stride, k_head_stride, head_dim)))
    return RELAXKV_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || (w_q_norm == nullptr) != (w_k_norm == nullptr)) return RELAXKV_ERR_INVALID_ARG;
  const relaxkv_status rc = check_rotary(rotary, positions, head_dim);
  if (rc != RELAXKV_OK) return rc;
  if (n_rows == 0) return RELAXKV_OK;
  DeviceStatus* st = status_word();
  const int sms = sm_count_of_current_device();
  if (!st || sms <= 0) return RELAXKV_ERR_CUDA;
  TurnArgs a = {};
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k);
  a.q_out = static_cast<uint16_t*>(q_out); a.k_out = static_cast<uint16_t*>(k_out);
  a.wq = static_cast<const uint16_t*>(w_q_norm); a.wk = static_cast<const uint16_t*>(w_k_norm);
  a.q_token = q_token_stride; a.q_head = (int)q_head_stride; a.k_token = k_token_stride; a.k_head = (int)k_head_stride;
  a.n_rows = n_rows; a.H = q ? n_q_heads : 0; a.Hkv = k ? n_kv_heads : 0; a.eps = eps;
  set_rotary(a, rotary, positions);
  const int per = rows_per_block(n_rows, a.H + a.Hkv, head_dim, sms);
  return cuda_ok(launch_turn_d<STORE_BF16>(head_dim, !rotary->interleaved, a, per, st, static_cast<cudaStream_t>(stream)));
}

extern "C" relaxkv_status relaxkv_append_quantized(
    const relaxkv_quantized_cache* store, const void* q, void* q_out, int64_t q_token_stride, int64_t q_head_stride, const void* k, const void* v,
    int64_t k_token_stride, int64_t k_head_stride, int64_t n_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* w_q_norm,
    const void* w_k_norm, float eps, const int32_t* positions, const relaxkv_rotary* rotary, const int32_t* slots, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_append_quantized");
  if (!slots || (q == nullptr) != (q_out == nullptr)) return RELAXKV_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || (q && n_q_heads < 1)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  relaxkv_status rc = check_quantized(store, n_kv_heads, head_dim);
  if (rc != RELAXKV_OK) return rc;
  if ((q && !bf16_rows_ok(q, q_out, q_token_stride, q_head_stride, head_dim)) || !bf16_rows_ok(k, v, k_token_stride, k_head_stride, head_dim)) return RELAXKV_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || (w_q_norm == nullptr) != (w_k_norm == nullptr)) return RELAXKV_ERR_INVALID_ARG;
  rc = check_rotary(rotary, positions, head_dim);
  if (rc != RELAXKV_OK) return rc;
  if (n_rows == 0) return RELAXKV_OK;
  DeviceStatus* st = status_word();
  const int sms = sm_count_of_current_device();
  if (!st || sms <= 0) return RELAXKV_ERR_CUDA;
  TurnArgs a = {};
  a.q = static_cast<const uint16_t*>(q); a.k = static_cast<const uint16_t*>(k); a.v = static_cast<const uint16_t*>(v);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.wq = static_cast<const uint16_t*>(w_q_norm); a.wk = static_cast<const uint16_t*>(w_k_norm);
  a.q_token = q_token_stride; a.q_head = (int)q_head_stride; a.k_token = k_token_stride; a.k_head = (int)k_head_stride;
  a.slots = slots; a.n_rows = n_rows; a.H = q ? n_q_heads : 0; a.Hkv = n_kv_heads; a.eps = eps;
  set_rotary(a, rotary, positions);
  set_store(a, store);
  const int per = rows_per_block(n_rows, a.H + 2 * a.Hkv, head_dim, sms);
  const bool half = rotary && rotary->dims > 0 && !rotary->interleaved;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (!q && !w_k_norm && a.part == 0)
    return cuda_ok(head_dim == 128 ? (store->type == RELAXKV_INT8 ? launch_store_plain<128, STORE_INT8>(a, per, st, s) : launch_store_plain<128, STORE_E4M3>(a, per, st, s))
                                   : (store->type == RELAXKV_INT8 ? launch_store_plain<64, STORE_INT8>(a, per, st, s) : launch_store_plain<64, STORE_E4M3>(a, per, st, s)));
  return cuda_ok(store->type == RELAXKV_INT8 ? launch_turn_d<STORE_INT8>(head_dim, half, a, per, st, s) : launch_turn_d<STORE_E4M3>(head_dim, half, a, per, st, s));
}

extern "C" relaxkv_status relaxkv_read_quantized(
    const relaxkv_quantized_cache* store, const int32_t* slots, int64_t n_rows, int32_t n_kv_heads, int32_t head_dim, const int32_t* positions,
    const relaxkv_rotary* rotary, void* k_out, void* v_out, int64_t token_stride, int64_t head_stride, relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_read_quantized");
  if (!slots || (positions == nullptr) != (rotary == nullptr)) return RELAXKV_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  relaxkv_status rc = check_quantized(store, n_kv_heads, head_dim);
  if (rc != RELAXKV_OK) return rc;
  if (!bf16_rows_ok(k_out, v_out, token_stride, head_stride, head_dim)) return RELAXKV_ERR_INVALID_ARG;
  rc = check_rotary(rotary, positions, head_dim);
  if (rc != RELAXKV_OK) return rc;
  if (n_rows == 0) return RELAXKV_OK;
  DeviceStatus* st = status_word();
  const int sms = sm_count_of_current_device();
  if (!st || sms <= 0) return RELAXKV_ERR_CUDA;
  TurnArgs a = {};
  a.k_out = static_cast<uint16_t*>(k_out); a.v_out = static_cast<uint16_t*>(v_out);
  a.k_token = token_stride; a.k_head = (int)head_stride;
  a.slots = slots; a.n_rows = n_rows; a.Hkv = n_kv_heads;
  set_rotary(a, rotary, positions);
  set_store(a, store);
  const int per = rows_per_block(n_rows, 2 * a.Hkv, head_dim, sms);
  const bool half = rotary && rotary->dims > 0 && !rotary->interleaved, int8 = store->type == RELAXKV_INT8;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a.part == 0)
    return cuda_ok(head_dim == 128 ? (int8 ? launch_read_plain<128, RELAXKV_INT8>(a, per, st, s) : launch_read_plain<128, RELAXKV_E4M3>(a, per, st, s))
                                   : (int8 ? launch_read_plain<64, RELAXKV_INT8>(a, per, st, s) : launch_read_plain<64, RELAXKV_E4M3>(a, per, st, s)));
  const cudaError_t e =
      head_dim == 128 ? (half ? (int8 ? launch_read<128, true, RELAXKV_INT8>(a, per, st, s) : launch_read<128, true, RELAXKV_E4M3>(a, per, st, s))
                              : (int8 ? launch_read<128, false, RELAXKV_INT8>(a, per, st, s) : launch_read<128, false, RELAXKV_E4M3>(a, per, st, s)))
                      : (half ? (int8 ? launch_read<64, true, RELAXKV_INT8>(a, per, st, s) : launch_read<64, true, RELAXKV_E4M3>(a, per, st, s))
                              : (int8 ? launch_read<64, false, RELAXKV_INT8>(a, per, st, s) : launch_read<64, false, RELAXKV_E4M3>(a, per, st, s)));
  return cuda_ok(e);
}
