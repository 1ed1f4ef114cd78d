// Internal: what the kernels of the attention over the 8-bit store share: arguments, the rows of a step, and how its work is dealt out.
#pragma once
#include "quantized_cache.cuh"
#include "sm100_ptx.cuh"

namespace relaxkv {

constexpr int kQaSeqsMost = 4096;
constexpr int kNoKey = -127;                     // exponent in shared memory of a token whose block does not exist

// A task that goes on in the next blocks, as the join finds it: blocks c0 to c1, its first row, KV head, columns, and which of them are written.
struct __align__(16) Chain { int c0, c1, row, head, cols; uint32_t live[4]; int none[3]; };

struct QuantAttnArgs {
  const uint16_t* q;
  uint16_t* out;
  float* lse_out;
  const uint8_t *k, *v;
  const int8_t *k_exp, *v_exp;
  const int *row_cu, *row_seq, *row_len, *table;
  float *part_o, *part_s;
  Chain* chain;
  long long block_stride, token_stride, head_stride, table_stride, n_rows;
  int table_width, n_seq, n_blocks, block_shift, max_len;
  int H, Hkv, G, rows_per_tile;
  int split;                             // blocks of a cluster that share a row tile and KV head
  int rows_at_once;                      // rows that a block, or cluster, looks through for the first ones of row tiles
  float scale_log2;
};

__device__ __forceinline__ float log2_of(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float one_over(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void copy_16(uint32_t dst, const void* src, int bytes) {       // bytes 16, or 0: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A maximum of nothing: no score lies below it, and what is taken from it stays a number (scores of -inf weigh nothing beside it, either).
constexpr float kNothing = -3.4028234663852886e38f;

// Rows and tokens of a sequence; rows 0: none to work on.
struct SeqRows { int first, n, len; };
// Rows first to end - 1 with the last one's length.
__device__ __forceinline__ SeqRows rows_with(const QuantAttnArgs& a, int seq, int first, int end, int len, bool tell, DeviceStatus* st) {
  SeqRows s = {first, 0, len};
  if (len < 0 || len > a.max_len || len > ((long long)a.table_width << a.block_shift)) {
    if (tell) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ATTN, len, seq);
    return s;
  }
  s.n = end - first;
  return s;
}
// guess_len: row_len[guess], read before it is known to be the last row's.
__device__ __forceinline__ SeqRows rows_of(const QuantAttnArgs& a, int seq, int guess, int guess_len, bool tell, DeviceStatus* st) {
  SeqRows s = {a.row_cu[seq], 0, 0};
  const int end = a.row_cu[seq + 1];
  if (s.first < 0 || end < s.first || end > a.n_rows) {
    if (tell) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ATTN, end, seq);
    return s;
  }
  if (end == s.first) return s;
  return rows_with(a, seq, s.first, end, end - 1 == guess ? guess_len : a.row_len[end - 1], tell, st);
}
// Tokens that a row of a sequence sees; -1: the row is left alone.
__device__ __forceinline__ int row_tokens(const QuantAttnArgs& a, int seq, const SeqRows& s, long long row, bool tell, DeviceStatus* st) {
  const int rs = a.row_seq[row], len = a.row_len[row];
  if (rs == seq && len >= 0 && len <= s.len) return len;
  if (tell && rs != -1) report(st, RELAXKV_ERR_BAD_INDEX, KID_QUANTIZED_ATTN, rs == seq ? len : rs, (int)row);
  return -1;
}


__device__ __forceinline__ long long quotient(long long a, long long b) {      // of numbers from 0 on; in 32 bits where these hold them
  return ((a | b) >> 31) == 0 ? (long long)((int)a / (int)b) : a / b;
}

// A block's share of a call.  The work - (sequence, KV head, row tile, TILE tokens), in this order - is a row of units, `per` of them to a block; a task, (sequence, KV head, row
// tile), counts UNITS more than it has tiles: the time that its start and end take.  Sequences are looked at by THREADS threads side by side.
template <int TILE, int UNITS, int LEAST, int THREADS>
struct Walk {
  struct Shared { long long sums[THREADS / 32], start; int seq; SeqRows s; };
  // the task that the block works on: tiles [j0, j1) of it
  int seq, hd, tile, j0, j1, tiles;
  SeqRows s;
  // units: where the block is, where its share ends; first ones of the sequence and the task
  long long f, f1, per, seq_start, task_start;

  static __device__ __forceinline__ int tiles_of(int len) { return max(1, (int)(((long long)len + TILE - 1) / TILE)); }      // (a sequence without tokens: for the zeros)
  __device__ __forceinline__ long long seq_units(const QuantAttnArgs& a) const {
    return (long long)((s.n + a.rows_per_tile - 1) / a.rows_per_tile) * a.Hkv * (tiles_of(s.len) + UNITS);
  }
  // The part of the task at f that belongs to this block (no tiles: its share ends before the task's first).
  __device__ __forceinline__ void cut(const QuantAttnArgs& a) {
    tiles = tiles_of(s.len);
    const int row_tiles = (s.n + a.rows_per_tile - 1) / a.rows_per_tile, task_units = tiles + UNITS;
    const long long task = quotient(f - seq_start, task_units);
    task_start = seq_start + task * task_units;
    hd = (int)quotient(task, row_tiles);
    tile = (int)(task - (long long)hd * row_tiles);
    const int o0 = (int)(f - task_start), o1 = (int)min((long long)task_units, o0 + (f1 - f));
    j0 = max(0, o0 - UNITS);
    j1 = max(0, o1 - UNITS);
    f += o1 - o0;
  }
  // The first task; false: the block has none.  For all threads of the block.
  __device__ __forceinline__ bool begin(const QuantAttnArgs& a, Shared& sh, DeviceStatus* st) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto units = [&](const SeqRows& x) -> long long {
      return x.n == 0 ? 0 : (long long)((x.n + a.rows_per_tile - 1) / a.rows_per_tile) * a.Hkv * (tiles_of(x.len) + UNITS);
    };
    const int per_thread = (a.n_seq + THREADS - 1) / THREADS, i0 = min(a.n_seq, tid * per_thread), i1 = tid < THREADS ? min(a.n_seq, i0 + per_thread) : i0;
    long long mine = 0;
    SeqRows x = {0, 0, 0};                               // (the last of this thread's sequences: the only one, mostly)
    const int each = (int)(a.n_rows / a.n_seq);          // where all sequences have as many rows, the last one's length comes with the row numbers
    for (int i = i0; i < i1; ++i) {
      const int guess = max(0, (i + 1) * each - 1);
      x = rows_of(a, i, guess, a.row_len[guess], blockIdx.x == 0, st);
      mine += units(x);
    }
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31 && tid < THREADS) sh.sums[warp] = upto;
    __syncthreads();
    long long all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) upto += sh.sums[w];
      all += sh.sums[w];
    }
    per = max(quotient(all + gridDim.x - 1, gridDim.x), (long long)LEAST);
    f = blockIdx.x * per;
    f1 = min(all, f + per);
    if (f >= f1) return false;
    if (tid < THREADS && f >= upto - mine && f < upto) {  // the share begins in one of this thread's sequences
      long long at = upto - mine;
      int i = i0;
      if (i + 1 < i1) {
        x = rows_of(a, i, -1, 0, false, st);
        for (long long n = units(x); f >= at + n && i + 1 < i1; n = units(x)) {
          at += n;
          x = rows_of(a, ++i, -1, 0, false, st);
        }
      }
      sh.seq = i;
      sh.start = at;
      sh.s = x;
    }
    __syncthreads();
    seq = sh.seq;
    seq_start = sh.start;
    s = sh.s;
    cut(a);
    return j1 > j0;
  }
  // On to the next task; false: the share ends.
  __device__ __forceinline__ bool next(const QuantAttnArgs& a, DeviceStatus* st) {
    if (f >= f1) return false;
    if (f - seq_start >= seq_units(a)) {
      seq_start = f;
      do s = rows_of(a, ++seq, -1, 0, false, st); while (s.n == 0 && seq + 1 < a.n_seq);      // (there is one: the share goes on)
      if (s.n == 0) return false;
    }
    cut(a);
    return j1 > j0;
  }
  __device__ __forceinline__ bool whole() const { return j0 == 0 && j1 == tiles; }
  __device__ __forceinline__ int slot() const { return 2 * (int)blockIdx.x + (j0 == 0 ? 1 : 0); }       // of a task's first part, of a later one
  // The blocks of a task that goes on in the next ones.
  __device__ __forceinline__ void blocks_of(int* c0, int* c1) const {
    *c0 = (int)quotient(task_start + UNITS, per);
    *c1 = (int)quotient(task_start + UNITS + tiles - 1, per);
  }
};

// The attention of many rows per sequence (quantized_rows_sm100.cu).
constexpr int kQrRows = 128, kQrBlocks = 148;      // (row, head) rows of a block; blocks that a call is cut into, at most
cudaError_t launch_quantized_rows(const QuantAttnArgs& a, int head_dim, int type, int sms, DeviceStatus* st, cudaStream_t stream);

}  // namespace relaxkv
