// Block tables and row metadata of a step, built on the GPU from request lengths (gfx950).
//
// With c_i cached and n_i new tokens of sequence i (blocks of 16 tokens):
//   have_i = ceil(c_i / 16), need_i = ceil((c_i + n_i) / 16) - have_i, base_i = sum_{j<i} need_j,
//   table[i][have_i + k] = free_blocks[used + base_i + k]           for k < need_i,
//   cu_i = sum_{j<i} n_j, and row r = cu_i + j is position p = c_i + j in slot
//   table[i][p / 16] * 16 + p % 16.
// Nothing here is bound by bytes (20 per row): the time is the launch and the chain of dependent
// steps, so one workgroup does it all (lengths, two scans, table entries, rows) where the rows
// are few; many rows go to a second launch that reads the tables and offsets that the first
// wrote. The checks come before the first write, so a refused step changes nothing but its status.
#include <limits.h>

#include "device_utils.h"
#include "internal.h"
#include "launch.h"

namespace pkv {
namespace {

constexpr int kFillThreads = 256;
constexpr int kFillRows = 1024;    // rows per workgroup of the second launch
constexpr int kFillSeqs = 4096;    // offsets it keeps in LDS (16 KB); above, it searches in memory

// The last i of 0 .. n - 1 with first[i] <= r (first ascending, first[0] <= r).
__device__ __forceinline__ int last_at_or_below(const int32_t* first, int n, int r) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Row r of the step: r < total belongs to a sequence, the others are padding.
__device__ __forceinline__ void fill_row(const ExtendArgs& a, const int32_t* cu, int total, int r) {
  int64_t slot = -1;
  int seq = -1, p = -1;
  if (r < total) {
    seq = last_at_or_below(cu, a.num_seqs, r);
    p = a.seq_lens[seq] - (cu[seq + 1] - r);
    const int blk = a.tables[(size_t)seq * a.max_blocks + p / kBlockSize];
    slot = (int64_t)blk * kBlockSize + p % kBlockSize;
  }
  if (a.slot_map != nullptr) a.slot_map[r] = slot;
  if (a.row_seq != nullptr) a.row_seq[r] = seq;
  if (a.positions != nullptr) a.positions[r] = p;
  if (a.row_lens != nullptr) a.row_lens[r] = p + 1;
}

// Exclusive scan over the workgroup's threads of two values at once; *ta, *tb: their totals.
template <int kThreads>
__device__ __forceinline__ void scan2(int& a, int& b, int* ta, int* tb, int (*sm)[2]) {
  constexpr int kWaves = kThreads / 64;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int a0 = a, b0 = b;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int ua = __shfl_up(a, off), ub = __shfl_up(b, off);
    if (lane >= off) {
      a += ua;
      b += ub;
    }
  }
  if (lane == 63) {
    sm[w][0] = a;
    sm[w][1] = b;
  }
  __syncthreads();
  a -= a0;
  b -= b0;
  *ta = *tb = 0;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    const int ka = sm[k][0], kb = sm[k][1];
    if (k < w) {
      a += ka;
      b += kb;
    }
    *ta += ka;
    *tb += kb;
  }
  __syncthreads();
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void extend_tables_kernel(ExtendArgs a, int fill_rows) {
  constexpr int kWaves = kThreads / 64;
  __shared__ int64_t sums[kWaves][2];
  __shared__ int scan[kWaves][2];
  __shared__ uint32_t flags[kWaves];
  __shared__ int32_t first[kThreads + 1];  // a chunk's base_i (then its end)
  __shared__ int32_t at[kThreads];         // table index of the sequence's first fresh block
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;

  // Totals and checks over every sequence, in 64 bits (lengths may be anything).
  int64_t rows = 0, blocks = 0;
  uint32_t bad = 0u;
  for (int i = t; i < a.num_seqs; i += kThreads) {
    const int64_t c = a.cached_lens[i], n = a.new_lens[i];
    const int64_t have = (c + kBlockSize - 1) / kBlockSize;
    const int64_t end = (c + n + kBlockSize - 1) / kBlockSize;
    if (c < 0 || n < 0 || c + n > INT_MAX) bad |= PKV_EXTEND_BAD_LENGTH;
    if (n > 0 && end > a.max_blocks) bad |= PKV_EXTEND_TABLE_FULL;
    rows += n;
    blocks += end - have;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    rows += __shfl_xor(rows, o);
    blocks += __shfl_xor(blocks, o);
    bad |= __shfl_xor(bad, o);
  }
  if (lane == 0) {
    sums[w][0] = rows;
    sums[w][1] = blocks;
    flags[w] = bad;
  }
  const int64_t used = *a.free_used;
  __syncthreads();
  rows = blocks = 0;
  bad = 0u;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    rows += sums[k][0];
    blocks += sums[k][1];
    bad |= flags[k];
  }
  if (!(bad & PKV_EXTEND_BAD_LENGTH)) {
    if (rows > a.max_rows) bad |= PKV_EXTEND_TOO_MANY_ROWS;
    if (used < 0 || used + blocks > a.num_free) bad |= PKV_EXTEND_OUT_OF_BLOCKS;
  }
  if (t == 0) {
    *a.status = (int32_t)bad;
    *a.free_used_out = (int32_t)(used + (bad ? 0 : blocks));
  }

  // Offsets, lengths and table entries, a chunk of sequences at a time.
  int rows0 = 0, blocks0 = 0;
  for (int i0 = 0; i0 < a.num_seqs; i0 += kThreads) {
    const int i = i0 + t;
    int c = 0, n = 0, have = 0, need = 0;
    if (i < a.num_seqs) {
      c = a.cached_lens[i];
      if (!bad) {
        n = a.new_lens[i];
        have = (int)(((int64_t)c + kBlockSize - 1) / kBlockSize);
        need = (int)(((int64_t)c + n + kBlockSize - 1) / kBlockSize) - have;
      }
    }
    int row = n, blk = need, trows, tblocks;
    scan2<kThreads>(row, blk, &trows, &tblocks, scan);
    if (i < a.num_seqs) {
      a.cu_new_lens[i] = rows0 + row;
      a.seq_lens[i] = c + n;
    }
    first[t] = blk;
    at[t] = have;
    __syncthreads();
    for (int e = t; e < tblocks; e += kThreads) {
      const int k = last_at_or_below(first, kThreads, e);
      a.tables[(size_t)(i0 + k) * a.max_blocks + at[k] + (e - first[k])] =
          a.free_blocks[used + blocks0 + e];
    }
    rows0 += trows;
    blocks0 += tblocks;
    __syncthreads();  // (first and at are written again)
  }
  if (t == 0) a.cu_new_lens[a.num_seqs] = rows0;
  if (fill_rows == 0) return;
  __syncthreads();  // the offsets, lengths and table entries of the other threads
  for (int r = t; r < a.max_rows; r += kThreads) fill_row(a, a.cu_new_lens, rows0, r);
}

__global__ __launch_bounds__(kFillThreads) void fill_rows_kernel(ExtendArgs a) {
  __shared__ int32_t cu_s[kFillSeqs + 1];
  const int total = a.cu_new_lens[a.num_seqs];
  const int32_t* cu = a.cu_new_lens;
  if (a.num_seqs <= kFillSeqs) {
    for (int i = threadIdx.x; i <= a.num_seqs; i += kFillThreads) cu_s[i] = a.cu_new_lens[i];
    __syncthreads();
    cu = cu_s;
  }
  const int r0 = blockIdx.x * kFillRows;
  for (int k = threadIdx.x; k < kFillRows && r0 + k < a.max_rows; k += kFillThreads)
    fill_row(a, cu, total, r0 + k);
}

}  // namespace

hipError_t launch_extend_tables(const ExtendArgs& a, hipStream_t stream) {
  const bool one = a.max_rows <= 4096;
  hipLaunchKernelGGL(extend_tables_kernel<1024>, dim3(1), dim3(1024), 0, stream, a, one ? 1 : 0);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || one) return err;
  hipLaunchKernelGGL(fill_rows_kernel, dim3((unsigned)((a.max_rows + kFillRows - 1) / kFillRows)),
                     dim3(kFillThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pkv
