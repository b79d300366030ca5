// Block tables and row metadata of a step, built on the GPU from request lengths (gfx950).
//
// With c_i cached and n_i new tokens of sequence i (blocks of 16 tokens):
//   have_i = ceil(c_i / 16), need_i = ceil((c_i + n_i) / 16) - have_i, base_i = sum_{j<i} need_j,
//   table[i][have_i + k] = free_blocks[used + base_i + k]           for k < need_i,
//   cu_i = sum_{j<i} n_j, and row r = cu_i + j is position p = c_i + j in slot
//   table[i][p / 16] * 16 + p % 16.
// Nothing here is bound by bytes (20 per row): the time is the launch and the chain of dependent
// steps, so one workgroup does it all (lengths, two scans, table entries, rows) where the rows
// are few; many rows go to a second launch of many workgroups, which reads the tables and offsets that
// the first wrote (the data do not force it: a new block's id stands in free_blocks, but each
// workgroup would scan the lengths for itself, and seq_lens may be cached_lens). Searches take a fixed number of steps, four of a thread's at a time. The checks come before
// the first write, so a refused step changes nothing but its status.
#include <limits.h>

#include "device_utils.h"
#include "internal.h"
#include "launch.h"
#include "wave_utils.h"

namespace pkv {
namespace {

constexpr int kFillThreads = 256;
constexpr int kFillRows = 1024;    // rows per workgroup of the second launch
constexpr int kFillSeqs = 4096;    // offsets it keeps in LDS (16 KB); above, it searches in memory

constexpr int kAtOnce = 4;         // searches of a thread side by side

// For each r[k]: the last i of 0 .. n - 1 with first[i] <= r[k] (first ascending, first[0] <= r[k]).
__device__ __forceinline__ void last_at_or_below(const int32_t* first, int n,
                                                 const int (&r)[kAtOnce], int (&at)[kAtOnce]) {
#pragma unroll
  for (int k = 0; k < kAtOnce; ++k) at[k] = 0;
  for (int step = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; step > 0; step >>= 1) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int to = at[k] + step;
      if (first[min(to, n - 1)] <= r[k] && to < n) at[k] = to;
    }
  }
}

// Rows r0, r0 + step, .. of the step below `end`: those below `total` belong to sequences, the others
// are padding.
__device__ __forceinline__ void fill_rows(const ExtendArgs& a, const int32_t* cu, int total,
                                          int64_t r0, int step, int64_t end) {
  for (int64_t b = r0; b < end; b += kAtOnce * step) {
    int r[kAtOnce], seq[kAtOnce], p[kAtOnce], blk[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) r[k] = (int)min(b + k * step, end - 1);
    last_at_or_below(cu, a.num_seqs, r, seq);
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      p[k] = r[k] < total ? a.seq_lens[seq[k]] - (cu[seq[k] + 1] - r[k]) : -1;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      blk[k] = r[k] < total ? a.tables[(size_t)seq[k] * a.max_blocks + p[k] / kBlockSize] : 0;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (b + k * step >= end) continue;
      const bool live = r[k] < total;
      if (a.slot_map != nullptr)
        a.slot_map[r[k]] = live ? (int64_t)blk[k] * kBlockSize + p[k] % kBlockSize : -1;
      if (a.row_seq != nullptr) a.row_seq[r[k]] = live ? seq[k] : -1;
      if (a.positions != nullptr) a.positions[r[k]] = p[k];
      if (a.row_lens != nullptr) a.row_lens[r[k]] = p[k] + 1;
    }
  }
}

// Exclusive scan over the workgroup's threads of two values at once; *ta, *tb: their totals.
template <int kThreads>
__device__ __forceinline__ void scan2(int& a, int& b, int* ta, int* tb, int (*sm)[2]) {
  constexpr int kWaves = kThreads / 64;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int ia = wave_scan(a), ib = wave_scan(b);
  if (lane == 63) {
    sm[w][0] = ia;
    sm[w][1] = ib;
  }
  __syncthreads();
  const int from = lane & 15;  // lane's wave
  const int sa = from < kWaves ? sm[from][0] : 0, sb = from < kWaves ? sm[from][1] : 0;
  *ta = row_all(sa, Add());
  *tb = row_all(sb, Add());
  a = ia - a + row_all(from < w ? sa : 0, Add());
  b = ib - b + row_all(from < w ? sb : 0, Add());
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void extend_tables_kernel(ExtendArgs a, int fill) {
  constexpr int kWaves = kThreads / 64;
  constexpr int kSums = 5;
  __shared__ int sums[kWaves][kSums];
  __shared__ int scan[kWaves][2];
  __shared__ int32_t first[kThreads];    // a chunk's base_i
  __shared__ int32_t at[kThreads];       // table index of the sequence's first fresh block
  __shared__ int32_t cu[kThreads + 1];   // offsets of a step of one chunk
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;

  // Totals and checks over every sequence, in 64 bits (lengths may be anything); the first chunk's
  // lengths are kept.
  int64_t rows = 0, blocks = 0;
  uint32_t bad = 0u;
  int c0 = 0, n0 = 0;
  for (int i = t; i < a.num_seqs; i += kThreads) {
    const int c32 = a.cached_lens[i], n32 = a.new_lens[i];
    if (i == t) {
      c0 = c32;
      n0 = n32;
    }
    const int64_t c = c32, n = n32;
    const int64_t have = (c + kBlockSize - 1) / kBlockSize;
    const int64_t end = (c + n + kBlockSize - 1) / kBlockSize;
    if (c < 0 || n < 0 || c + n > INT_MAX) bad |= PKV_EXTEND_BAD_LENGTH;
    if (n > 0 && end > a.max_blocks) bad |= PKV_EXTEND_TABLE_FULL;
    rows += n;
    blocks += end - have;
  }
  const int64_t used = *a.free_used;
  // sums in two parts of 32 bits (a thread's, cut at 2^34, is past every limit then)
  auto cut = [](int64_t v) { return v < 0 ? 0 : v >> 34 != 0 ? (int64_t)1 << 34 : v; };
  rows = cut(rows);
  blocks = cut(blocks);
  int part[kSums] = {(int)(rows & 32767), (int)(rows >> 15), (int)(blocks & 32767),
                     (int)(blocks >> 15), (int)bad};
#pragma unroll
  for (int k = 0; k < kSums; ++k) part[k] = k < 4 ? wave_all(part[k], Add()) : wave_all(part[k], Or());
  if (lane == 0) {
#pragma unroll
    for (int k = 0; k < kSums; ++k) sums[w][k] = part[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    const int x = (lane & 15) < kWaves ? sums[lane & 15][k] : 0;
    part[k] = k < 4 ? row_all(x, Add()) : row_all(x, Or());
  }
  rows = ((int64_t)part[1] << 15) + part[0];
  blocks = ((int64_t)part[3] << 15) + part[2];
  bad = (uint32_t)part[4];
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
    int c = c0, n = n0, have = 0, need = 0;
    if (i0 > 0 && i < a.num_seqs) {
      c = a.cached_lens[i];
      n = a.new_lens[i];
    }
    if (i >= a.num_seqs || bad) n = 0;
    if (i < a.num_seqs && !bad) {
      have = (int)(((int64_t)c + kBlockSize - 1) / kBlockSize);
      need = (int)(((int64_t)c + n + kBlockSize - 1) / kBlockSize) - have;
    }
    int row = n, blk = need, trows, tblocks;
    scan2<kThreads>(row, blk, &trows, &tblocks, scan);
    if (i < a.num_seqs) {
      a.cu_new_lens[i] = rows0 + row;
      a.seq_lens[i] = c + n;
    }
    cu[t] = rows0 + row;
    first[t] = blk;
    at[t] = have;
    __syncthreads();
    for (int b = t; b < tblocks; b += kAtOnce * kThreads) {
      int e[kAtOnce], k[kAtOnce], id[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        e[j] = min(b + j * kThreads, tblocks - 1);
        id[j] = a.free_blocks[used + blocks0 + e[j]];
      }
      last_at_or_below(first, kThreads, e, k);
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (b + j * kThreads < tblocks)
          a.tables[(size_t)(i0 + k[j]) * a.max_blocks + at[k[j]] + (e[j] - first[k[j]])] = id[j];
    }
    rows0 += trows;
    blocks0 += tblocks;
    if (i0 + kThreads < a.num_seqs) __syncthreads();  // (first, at and scan are written again)
  }
  if (t == 0) {
    a.cu_new_lens[a.num_seqs] = rows0;
    cu[min(a.num_seqs, kThreads)] = rows0;
  }
  if (fill == 0) return;
  __syncthreads();  // the offsets, lengths and table entries of the other threads
  if (a.num_seqs <= kThreads) fill_rows(a, cu, rows0, t, kThreads, a.max_rows);
  else fill_rows(a, a.cu_new_lens, rows0, t, kThreads, a.max_rows);
}

__global__ __launch_bounds__(kFillThreads) void fill_rows_kernel(ExtendArgs a) {
  __shared__ int32_t cu[kFillSeqs + 1];
  const int total = a.cu_new_lens[a.num_seqs];
  const int64_t r0 = (int64_t)blockIdx.x * kFillRows, end = min(r0 + kFillRows, (int64_t)a.max_rows);
  if (a.num_seqs <= kFillSeqs && r0 < total) {
    for (int i = threadIdx.x; i <= a.num_seqs; i += kFillThreads) cu[i] = a.cu_new_lens[i];
    __syncthreads();
    fill_rows(a, cu, total, r0 + threadIdx.x, kFillThreads, end);
  } else {
    fill_rows(a, a.cu_new_lens, total, r0 + threadIdx.x, kFillThreads, end);
  }
}

}  // namespace

hipError_t launch_extend_tables(const ExtendArgs& a, hipStream_t stream) {
  // One launch up to 4096 rows (a second one costs more than its workgroups save), and four waves
  // instead of sixteen where these are enough: a decode step of 64 sequences 3.9 us against 5.8.
  const bool one = a.max_rows <= 4096, small = a.num_seqs <= 256 && a.max_rows <= 1024;
  hipLaunchKernelGGL(small ? extend_tables_kernel<256> : extend_tables_kernel<1024>, dim3(1),
                     dim3(small ? 256 : 1024), 0, stream, a, one ? 1 : 0);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || one) return err;
  hipLaunchKernelGGL(fill_rows_kernel, dim3((unsigned)((a.max_rows + kFillRows - 1) / kFillRows)),
                     dim3(kFillThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pkv
