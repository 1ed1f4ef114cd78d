// Block tables and slot maps of a step over continuations, from the sequences' lengths (relaxkv_build_block_tables).
//
// Three running sums over the sequences decide everything: rows appended, blocks needed, blocks given back.  They are a few thousand
// numbers, so every block of the launch computes them for itself from the lengths (all in L2) and then writes its share of the outputs: rows,
// new table entries and what is left of the released blocks, each found by bisection in the sums.  No block waits for another and there is one
// launch.  Entries that are read (blocks a sequence has, free blocks below n_free) are never entries that are written, which is what lets the
// blocks of the launch run in any order and the call be repeated.
#include "continuations.cuh"
#include <algorithm>

namespace relaxkv {

constexpr int kTabMaxSeq = 4096;

struct TableArgs {
  int n_seq, block_size, free_capacity, table_width;
  long long table_stride, n_rows;
  const int *seq_len, *new_len, *seq_base, *n_free;
  int *free_blocks, *table, *seq_len_out, *n_free_out, *row_cu, *row_seq, *row_pos, *row_len, *row_slot;
};

__device__ __forceinline__ int blocks_of(int tokens, int shift) { return (int)(((long long)tokens + (1 << shift) - 1) >> shift); }

// The segment of cu[0 .. n] that x lies in: the last i with cu[i] <= x (empty segments are passed over).
__device__ __forceinline__ int bisect(const int* cu, int n, int x) {
  int lo = 0;
  for (int hi = n; hi - lo > 1;) { const int mid = (lo + hi) >> 1; if (cu[mid] <= x) lo = mid; else hi = mid; }
  return lo;
}

// PER: sequences of a thread, at most.
template <int THREADS, int PER>
__global__ void __launch_bounds__(THREADS)
block_tables_kernel(const TableArgs a, DeviceStatus* st) {
  extern __shared__ int cu_s[];
  int *rows_cu = cu_s, *need_cu = cu_s + a.n_seq + 1, *back_cu = need_cu + a.n_seq + 1, *had_s = back_cu + a.n_seq + 1;
  __shared__ long long warp_rows[THREADS / 32];
  __shared__ int warp_need[THREADS / 32], warp_back[THREADS / 32];
  griddep_launch();
  griddep_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = THREADS / 32;
  const int shift = 31 - __clz(a.block_size);
  const bool teller = blockIdx.x == 0;
  const int per = (a.n_seq + THREADS - 1) / THREADS, first = min(a.n_seq, tid * per), last = min(a.n_seq, first + per);
  const long long room = min((long long)a.table_width << shift, 0x7fffffffLL);
  const int n_free = *a.n_free;
  // lengths and requests by way of shared memory (the requests in the place of a sum that comes later), then a thread's own in registers: what
  // one asks for and cannot have counts as nothing
  for (int i = tid; i < a.n_seq; i += THREADS) { had_s[i] = a.seq_len[i]; rows_cu[i] = a.new_len[i]; }
  __syncthreads();
  int had_[PER], rows_[PER], need_[PER], back_[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    had_[e] = first + e < last ? had_s[first + e] : 0;
    rows_[e] = first + e < last ? rows_cu[first + e] : 0;
  }
  // ---- the sums: this thread's sequences, its warp's threads, the block's warps ----
  long long rows_t = 0;
  int need_t = 0, back_t = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    need_[e] = back_[e] = 0;
    if (e >= per) continue;                             // (the same for all threads)
    const int len = had_[e], add = rows_[e];
    const bool ok = len >= 0 && len <= room && add <= a.n_rows && (long long)len + max(add, 0) <= room;
    if (!ok && teller) report(st, RELAXKV_ERR_BAD_INDEX, KID_TABLES, first + e, add);
    rows_[e] = ok ? max(add, 0) : 0;
    need_[e] = ok && add > 0 ? blocks_of(len + add, shift) - blocks_of(len, shift) : 0;
    back_[e] = ok && add < 0 ? blocks_of(len, shift) : 0;
    rows_t += rows_[e]; need_t += need_[e]; back_t += back_[e];
  }
  long long rows_x = rows_t;
  int need_x = need_t, back_x = back_t;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long r = __shfl_up_sync(0xffffffffu, rows_x, o);
    const int n = __shfl_up_sync(0xffffffffu, need_x, o), k = __shfl_up_sync(0xffffffffu, back_x, o);
    if (lane >= o) { rows_x += r; need_x += n; back_x += k; }
  }
  if (lane == 31) { warp_rows[warp] = rows_x; warp_need[warp] = need_x; warp_back[warp] = back_x; }
  __syncthreads();
  long long rows_before, total_rows;
  int need_before, back_before, total_need, total_back;
  {                                                     // every warp adds up the warps' sums, a warp per lane
    long long r = lane < n_warps ? warp_rows[lane] : 0;
    int n = lane < n_warps ? warp_need[lane] : 0, k = lane < n_warps ? warp_back[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long r2 = __shfl_up_sync(0xffffffffu, r, o);
      const int n2 = __shfl_up_sync(0xffffffffu, n, o), k2 = __shfl_up_sync(0xffffffffu, k, o);
      if (lane >= o) { r += r2; n += n2; k += k2; }
    }
    total_rows = __shfl_sync(0xffffffffu, r, 31);
    total_need = __shfl_sync(0xffffffffu, n, 31);
    total_back = __shfl_sync(0xffffffffu, k, 31);
    rows_before = warp == 0 ? 0 : __shfl_sync(0xffffffffu, r, max(warp - 1, 0));
    need_before = warp == 0 ? 0 : __shfl_sync(0xffffffffu, n, max(warp - 1, 0));
    back_before = warp == 0 ? 0 : __shfl_sync(0xffffffffu, k, max(warp - 1, 0));
  }
  // (the sums of the blocks fit 32 bits: a table of 2^31 entries or more is refused on the host)
  const bool nothing = n_free < 0 || (long long)n_free + total_back > a.free_capacity;
  const bool full = !nothing && (total_rows > a.n_rows || total_need > n_free + total_back);
  if (teller && tid == 0 && (nothing || full)) report(st, RELAXKV_ERR_BAD_INDEX, KID_TABLES, nothing ? -1 : -2, nothing ? n_free : total_need);
  const bool grow = !nothing && !full;
  if (nothing) total_back = 0;
  if (!grow) { total_rows = 0; total_need = 0; }
  {
    long long rows_at = rows_before + rows_x - rows_t;
    int need_at = need_before + need_x - need_t, back_at = back_before + back_x - back_t;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = first + e;
      if (i >= last) break;
      rows_cu[i] = grow ? (int)rows_at : 0;
      need_cu[i] = grow ? need_at : 0;
      back_cu[i] = nothing ? 0 : back_at;
      rows_at += rows_[e]; need_at += need_[e]; back_at += back_[e];
      if (teller) {
        a.row_cu[i] = rows_cu[i];
        a.seq_len_out[i] = !nothing && back_[e] > 0 ? 0 : had_[e] + (grow ? rows_[e] : 0);
      }
    }
  }
  if (tid == 0) { rows_cu[a.n_seq] = (int)total_rows; need_cu[a.n_seq] = total_need; back_cu[a.n_seq] = total_back; }
  if (teller && tid == 0) { a.row_cu[a.n_seq] = (int)total_rows; *a.n_free_out = nothing ? n_free : n_free + total_back - total_need; }
  __syncthreads();
  // ---- the outputs ----
  const int top = n_free + total_back;
  auto released = [&](int j) -> const int* {     // where the j-th released block's number stands
    const int i = bisect(back_cu, a.n_seq, j);
    return a.table + i * a.table_stride + (j - back_cu[i]);
  };
  auto taken = [&](int j) -> const int* {        // and that of the j-th block of the stack from its end
    const int at = top - 1 - j;
    return at < n_free ? a.free_blocks + at : released(at - n_free);
  };
  const long long step = (long long)gridDim.x * THREADS, me = (long long)blockIdx.x * THREADS + tid;
  for (long long j = me; j < total_need; j += step) {
    const int i = bisect(need_cu, a.n_seq, (int)j);
    a.table[i * a.table_stride + blocks_of(had_s[i], shift) + ((int)j - need_cu[i])] = *taken((int)j);
  }
  for (long long j = n_free + me; j < top - total_need; j += step) a.free_blocks[j] = *released((int)j - n_free);
  for (long long r = me; r < a.n_rows; r += step) {
    int seq = -1, pos = 0, len = 0, slot = -1;
    if (r < total_rows) {
      seq = bisect(rows_cu, a.n_seq, (int)r);
      const int had = had_s[seq], at = had + ((int)r - rows_cu[seq]), have = blocks_of(had, shift), j = at >> shift;
      const int block = *(j < have ? a.table + seq * a.table_stride + j : taken(need_cu[seq] + (j - have)));
      pos = (a.seq_base ? a.seq_base[seq] : 0) + at;
      len = at + 1;
      if (block >= 0 && ((long long)block << shift) <= 0x7fffffffLL - (1 << shift)) slot = (int)(((unsigned)block << shift) + (at & ((1 << shift) - 1)));
      else report(st, RELAXKV_ERR_BAD_INDEX, KID_TABLES, seq, block);
    }
    a.row_seq[r] = seq;
    a.row_pos[r] = pos;
    a.row_len[r] = len;
    a.row_slot[r] = slot;
  }
}

}  // namespace relaxkv

using namespace relaxkv;

extern "C" relaxkv_status relaxkv_build_block_tables(
    int32_t n_seq, int32_t block_size, const int32_t* seq_len, const int32_t* new_len, const int32_t* seq_base, int32_t* free_blocks,
    int32_t free_capacity, const int32_t* n_free, int32_t* block_table, int32_t table_width, int64_t table_stride, int64_t n_rows,
    int32_t* seq_len_out, int32_t* n_free_out, int32_t* row_cu, int32_t* row_seq, int32_t* row_pos, int32_t* row_len, int32_t* row_slot,
    relaxkv_stream stream) {
  RELAXKV_RANGE("relaxkv_build_block_tables");
  if (!seq_len || !new_len || !free_blocks || !n_free || !block_table || !seq_len_out || !n_free_out || !row_cu) return RELAXKV_ERR_INVALID_ARG;
  if (n_seq < 1 || n_rows < 0 || free_capacity < 0 || table_width < 1 || table_stride < table_width) return RELAXKV_ERR_INVALID_ARG;
  if (n_rows > 0 && (!row_seq || !row_pos || !row_len || !row_slot)) return RELAXKV_ERR_INVALID_ARG;
  // the blocks of the launch read these while others may already write the results
  if (seq_len_out == seq_len || seq_len_out == new_len || n_free_out == n_free) return RELAXKV_ERR_INVALID_ARG;
  if (!block_size_ok(block_size) || n_seq > kTabMaxSeq) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  if (n_rows > 0x7fffffffLL || (long long)n_seq * table_width > 0x7fffffffLL) return RELAXKV_ERR_UNSUPPORTED_SHAPE;
  DeviceStatus* st = status_word();
  const int sms = sm_count_of_current_device();
  if (!st || sms <= 0) return RELAXKV_ERR_CUDA;
  const TableArgs a = {n_seq, block_size, free_capacity, table_width, (long long)table_stride, (long long)n_rows, seq_len, new_len, seq_base, n_free,
                       free_blocks, block_table, seq_len_out, n_free_out, row_cu, row_seq, row_pos, row_len, row_slot};
  // One block per SM at most: more of them repeat the sums for less than they bring (452 K rows of 1600 sequences: 12.1 us with two of 512 threads, 11.8
  // so; a million rows of 4096 17.9 and 14.0; 320 K rows of 64 5.3 so, 6.8 with four of 256).  Few rows: a block for the sums, as small as the sequences
  // allow (graph replay, 64 sequences of a token each: 2.9 us with 256 threads, 3.9 with 1024; 500 of four tokens 5.2 with 512, 6.4).
  const int threads = n_rows > 256LL * sms || n_seq > 1024 ? 1024 : n_seq > 256 ? 512 : 256;
  auto kern = threads == 256 ? block_tables_kernel<256, 1> : threads == 512 ? block_tables_kernel<512, 2> : block_tables_kernel<1024, 4>;
  const size_t smem = 4 * 4 * (size_t)(n_seq + 1);
  if (threads == 1024) {                                 // (the others stay below what a launch may have without asking)
    static std::atomic<int> attr_done[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return RELAXKV_ERR_CUDA;
    if (!attr_done[dev].load(std::memory_order_acquire)) {
      if (cudaFuncSetAttribute(block_tables_kernel<1024, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, 4 * 4 * (kTabMaxSeq + 1)) != cudaSuccess)
        return RELAXKV_ERR_CUDA;
      attr_done[dev].store(1, std::memory_order_release);
    }
  }
  const long long blocks = std::max<long long>(1, std::min<long long>(sms, (n_rows + threads - 1) / threads));
  return cuda_ok(launch_chained(kern, dim3((unsigned)blocks), (unsigned)threads, smem, static_cast<cudaStream_t>(stream), a, st));
}
