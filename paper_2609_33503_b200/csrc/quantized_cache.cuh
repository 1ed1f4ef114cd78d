// Internal: the 8-bit store: argument checks, and how its bytes become numbers.
#pragma once
#include "continuations.cuh"
#include <cuda_fp16.h>

namespace relaxkv {

constexpr int kExpNone = -128;         // exponent of a token and head whose elements are NaN
constexpr int kExpLeast = -100;

inline relaxkv_status check_quantized(const relaxkv_quantized_cache* c, int32_t n_kv_heads, int32_t head_dim) {
  if (!c || !c->k || !c->v || !c->k_exp || !c->v_exp) return RELAXKV_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_exp) || !aligned16(c->v_exp)) return RELAXKV_ERR_INVALID_ARG;
  if (c->type != RELAXKV_INT8 && c->type != RELAXKV_E4M3) return RELAXKV_ERR_INVALID_ARG;
  if ((head_dim != 64 && head_dim != 128) || !block_size_ok(c->block_size)) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (n_kv_heads < 1 || n_kv_heads != c->n_kv_heads) return RELAXKV_ERR_INVALID_ARG;
  if (c->n_blocks < 1 || (long long)c->n_blocks * c->block_size > 0x7fffffffLL) return RELAXKV_ERR_INVALID_ARG;     // slots are int32
  if (c->block_stride < head_dim || c->token_stride < head_dim || c->head_stride < head_dim) return RELAXKV_ERR_INVALID_ARG;
  if (c->block_stride % 16 || c->token_stride % 16 || c->head_stride % 16 || c->head_stride > 0x7fffffff) return RELAXKV_ERR_INVALID_ARG;
  return RELAXKV_OK;
}

// 2^e for an exponent of the store; NaN for kExpNone.
__device__ __forceinline__ float exp_scale(int e) {
  return e == kExpNone ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(e + 127) << 23);
}

// Two of the four int8 values of w (already with their sign bits flipped: w ^ 0x80808080) as fp16: 0x6400 | byte is 1024 + byte, exactly.  sel: 0x4140
// for bytes 0 and 1, 0x4342 for 2 and 3, 0x4240 and 0x4341 for the even and the odd ones.
template <uint32_t SEL>
__device__ __forceinline__ uint32_t int8_to_half2(uint32_t flipped) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(flipped), "r"(0x64646464u), "n"(SEL));
  asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(r) : "r"(0x64806480u));          // 1024 + 128
  return r;
}
// The two e4m3 values of the low (hi = 0) or high half of w as fp16, exactly.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t w, int hi) {
  uint32_t r;
  const uint16_t h = (uint16_t)(hi ? w >> 16 : w & 0xffffu);
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(h));
  return r;
}

}  // namespace relaxkv
