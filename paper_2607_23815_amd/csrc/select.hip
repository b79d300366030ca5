// The choice of blocks for sparse attention (gfx950). For a row (one query token) of g heads per kv
// head and a block whose keys lie within [lo, hi] dim by dim, the score
//   s = max_h sum_d max(q_hd hi_d, q_hd lo_d)
// is the most that a key of the block could score for any of the group's heads. The first `sink`
// and the last `recent` blocks of the row are always chosen, the others by score, ties by the
// lowest index, `blocks` in all.
//
// With q+ = max(q, 0) and q- = min(q, 0) the inner sum is q+ . hi + q- . lo: a matrix product over
// 2 D dims, which the matrix cores take in bf16 with 32-bit sums (score_kernel). Those sums carry
// rounding errors, and a choice must not depend on them: with |s - exact| <= err for every block,
// blocks more than 2 err above (below) the last chosen score are in (out) for certain, and the few
// between are scored again in 64 bits (select_kernel), where the products of bf16 values are exact.
//
// One row per sequence is bound by reading the bounds (4 D bytes per block and kv head).
#include <math.h>

#include "device_utils.h"
#include "launch.h"

namespace pkv {
namespace {

constexpr int kScoreWaves = 4;
constexpr int kSelThreads = 256;
constexpr int kSelWaves = kSelThreads / 64;
constexpr int kBins = 2048;
constexpr int kCand = 512;  // blocks near the border that are ranked in LDS

// The row's blocks (those with a visible key), as both kernels count them.
__device__ __forceinline__ int row_blocks(const SelectArgs& a, int64_t row) {
  const int len = min(a.row_lens[row], a.max_len);
  return len <= 0 ? 0 : min((int)(((int64_t)len + kBlockSize - 1) / kBlockSize), a.max_blocks);
}
__device__ __forceinline__ int row_sequence(const SelectArgs& a, int64_t row) {
  const int s = a.row_seq != nullptr ? a.row_seq[row] : (int)row;
  return s >= 0 && s < a.num_seqs ? s : -1;
}

// A wave per 16 blocks of a (row, kv head), a workgroup per 64: A = q (16 heads x 32 dims), B = bounds (32 dims x 16
// blocks), so lane (block l % 16, group l / 16) ends with the scores of heads 4 (l / 16) + 0..3.
template <int D>
__device__ __forceinline__ void score_tile(const SelectArgs& a, int64_t work, int chunks) {
  constexpr int KK = D / 32;
  const int64_t item = work / chunks;  // (row, kv head)
  const int64_t row = item / a.hkv;
  const int kvh = (int)(item % a.hkv);
  const int n = row_blocks(a, row);
  const int seq = row_sequence(a, row);
  const int tile = (int)(work % chunks) * kScoreWaves + (threadIdx.x >> 6);
  if (seq < 0 || n <= a.blocks || tile * 16 >= n) return;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int g = a.hq / a.hkv;
  const int b = min(tile * 16 + col, n - 1);
  const int id = a.tables[(size_t)seq * a.max_blocks + b];
  const uint16_t* box = a.bounds + ((size_t)(id < 0 || id >= a.num_blocks ? 0 : id) * a.hkv + kvh) * 2 * D;
  const uint16_t* q = a.q + ((size_t)row * a.hq + kvh * g + col) * D;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  uint32_t most = 0u;  // the largest |bound| of this lane, as bf16 bits
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      const int d = kk * 32 + grp * 8;
      u32x4 qv = {0u, 0u, 0u, 0u};
      if (col < g) qv = ld16(q + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // the positive parts, then the negative ones
        const uint32_t lo = qv[e] & 0xFFFFu, hi = qv[e] >> 16;
        const uint32_t keep_lo = (lo >> 15) == (uint32_t)side ? lo : 0u;
        const uint32_t keep_hi = (hi >> 15) == (uint32_t)side ? hi : 0u;
        qv[e] = keep_lo | keep_hi << 16;
      }
      const u32x4 bv = ld16(box + side * D + d);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        most = max(most, max(bv[e] & 0x7FFFu, bv[e] >> 16 & 0x7FFFu));
      s = mfma16(as_bf16x8(qv), as_bf16x8(bv), s);
    }
  }
  float best = -INFINITY;
  bool odd = false;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (4 * grp + r < g) {
      best = fmaxf(best, s[r]);
      odd |= !isfinite(s[r]);
    }
  }
  if (odd) best = INFINITY;
  best = fmaxf(best, __shfl_xor(best, 16));
  best = fmaxf(best, __shfl_xor(best, 32));
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
  if (grp == 0 && tile * 16 + col < n) a.scores[item * a.stride + tile * 16 + col] = best;
  if (lane == 0) a.tile_most[item * (a.stride / 16) + tile] = __uint_as_float(most << 16);
}

template <int D>
__global__ __launch_bounds__(64 * kScoreWaves) void score_kernel(const SelectArgs a, int chunks,
                                                                 int64_t total) {
  for (int64_t work = blockIdx.x; work < total; work += gridDim.x) score_tile<D>(a, work, chunks);
}

template <typename T, typename F>
__device__ __forceinline__ T wg_reduce(T v, F op, T* sm) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = op(v, (T)__shfl_xor(v, o));
  __syncthreads();  // (sm's readers of the last call)
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
  __syncthreads();
  v = sm[0];
#pragma unroll
  for (int k = 1; k < kSelWaves; ++k) v = op(v, sm[k]);
  return v;
}

// A score in 64 bits by one wave, as a key whose unsigned order is the scores' order (a score that
// is not finite counts as +infinity). Never 0 and never ~0.
template <int D>
__device__ __forceinline__ uint64_t exact_key(const SelectArgs& a, const uint16_t* q, int g,
                                              const int32_t* table, int kvh, int b) {
  constexpr int PER = D / 64;
  const int lane = threadIdx.x & 63;
  const int id = table[b];
  const uint16_t* box = a.bounds + ((size_t)(id < 0 || id >= a.num_blocks ? 0 : id) * a.hkv + kvh) * 2 * D;
  double hi[PER], lo[PER];
  bool odd = false;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const float x = __uint_as_float((uint32_t)box[lane * PER + e] << 16);
    const float y = __uint_as_float((uint32_t)box[D + lane * PER + e] << 16);
    odd |= !isfinite(x) || !isfinite(y);
    hi[e] = x;
    lo[e] = y;
  }
  double best = -INFINITY;
  for (int h = 0; h < g; ++h) {
    double s = 0.;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const float x = __uint_as_float((uint32_t)q[h * D + lane * PER + e] << 16);
      odd |= !isfinite(x);
      s += (double)x * (x > 0.f ? hi[e] : lo[e]);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o);
    best = fmax(best, s);
  }
  if (__builtin_amdgcn_ballot_w64(odd) != 0) best = INFINITY;
  best += 0.;  // (-0 becomes +0: equal scores, equal keys)
  const uint64_t u = (uint64_t)__double_as_longlong(best);
  return u >> 63 ? ~u : u | 1ull << 63;
}

// One workgroup per (row, kv head).
template <int D>
__global__ __launch_bounds__(kSelThreads) void select_kernel(const SelectArgs a) {
  __shared__ uint32_t chosen[kSelectMaxBlocks / 32];
  __shared__ uint32_t bins[kBins];
  __shared__ uint64_t cand_key[kCand];
  __shared__ int cand_at[kCand];
  __shared__ float smf[kSelWaves];
  __shared__ int smi[kSelWaves];
  __shared__ int num_cand, pivot;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int64_t item = blockIdx.x;
  const int64_t row = item / a.hkv;
  const int kvh = (int)(item % a.hkv);
  const int seq = row_sequence(a, row);
  if (seq < 0) return;  // a padding row
  const int n = row_blocks(a, row);
  int32_t* sel = a.sel + item * a.blocks;
  if (n <= a.blocks) {  // every block
    for (int k = t; k < a.blocks; k += kSelThreads) sel[k] = k < n ? k : -1;
    return;
  }
  const int first = a.sink, last = n - a.recent;  // [first, last) goes by score
  const int want = a.blocks - a.sink - a.recent;
  float* score = a.scores + item * a.stride;
  float* low = a.low + item * a.stride;
  const int32_t* table = a.tables + (size_t)seq * a.max_blocks;
  const int g = a.hq / a.hkv;
  const uint16_t* q = a.q + ((size_t)row * a.hq + kvh * g) * D;

  for (int k = t; k < (n + 31) / 32; k += kSelThreads) chosen[k] = 0u;
  if (t == 0) num_cand = 0;
  for (int k = t; k < kBins; k += kSelThreads) bins[k] = 0u;
  __syncthreads();
  auto choose = [&](int b) { atomicOr(&chosen[b >> 5], 1u << (b & 31)); };
  for (int k = t; k < a.sink + a.recent; k += kSelThreads)
    choose(k < a.sink ? k : n - a.recent + (k - a.sink));

  if (want > 0) {
    // the error of a 32-bit score: 2 D products summed in some order, each addition off by at most
    // 2^-23 of the sum of their magnitudes, |q|_1 max |bound|; tiny values may count as zeros
    float norm = 0.f, qmost = 0.f;
    for (int h = w; h < g; h += kSelWaves) {
      float s = 0.f, m = 0.f;
      for (int d = lane; d < D; d += 64) {
        const float x = fabsf(__uint_as_float((uint32_t)q[h * D + d] << 16));
        s += x;
        m = fmaxf(m, x);
      }
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) {
        s += __shfl_xor(s, o);
        m = fmaxf(m, __shfl_xor(m, o));
      }
      norm = fmaxf(norm, s);
      qmost = fmaxf(qmost, m);
    }
    auto maxf = [](float x, float y) { return fmaxf(x, y); };
    auto minf = [](float x, float y) { return fminf(x, y); };
    auto addi = [](int x, int y) { return x + y; };
    norm = wg_reduce(norm, maxf, smf);
    qmost = wg_reduce(qmost, maxf, smf);
    float most = 0.f;
    for (int k = t; k < (n + 15) / 16; k += kSelThreads)
      most = fmaxf(most, a.tile_most[item * (a.stride / 16) + k]);
    most = wg_reduce(most, maxf, smf);
    const float tiny = 0x1p-118f;
    const float err2 = 2.f * (0x1p-15f * 1.01f * norm * most + tiny * (1.f + qmost + most));

    // how the scores spread: a histogram between the least and the largest finds the bin of the
    // last chosen one
    float mn = INFINITY, mx = -INFINITY;
    for (int b = first + t; b < last; b += kSelThreads) {
      mn = fminf(mn, score[b]);
      mx = fmaxf(mx, score[b]);
    }
    mn = wg_reduce(mn, minf, smf);
    mx = wg_reduce(mx, maxf, smf);
    const float range = mx - mn;
    bool slow = !(isfinite(err2) && isfinite(mn) && isfinite(mx) && isfinite(range));
    const float per = range > 0.f ? (kBins - 1) / range : 0.f;
    auto bin_of = [&](float s) { return min((int)((s - mn) * per), kBins - 1); };
    float lo = 0.f, hi = 0.f;
    if (!slow) {
      for (int b = first + t; b < last; b += kSelThreads) atomicAdd(&bins[bin_of(score[b])], 1u);
      __syncthreads();
      // thread t counts bins [8 (255 - t), 8 (255 - t) + 8): a scan from the top
      constexpr int kPer = kBins / kSelThreads;
      int mine = 0;
      for (int k = 0; k < kPer; ++k) mine += bins[(kSelThreads - 1 - t) * kPer + k];
      int incl = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(incl, o);
        if (lane >= o) incl += u;
      }
      if (lane == 63) smi[w] = incl;
      __syncthreads();
      for (int k = 0; k < w; ++k) incl += smi[k];
      if (incl - mine < want && want <= incl) {  // (one thread)
        int left = want - (incl - mine), k = kPer - 1;
        while (left > (int)bins[(kSelThreads - 1 - t) * kPer + k])
          left -= bins[(kSelThreads - 1 - t) * kPer + k--];
        pivot = (kSelThreads - 1 - t) * kPer + k;
      }
      __syncthreads();
      // the scores of that bin lie in [lo, hi]: fewer than `want` lie above, at least from lo on
      lo = INFINITY;
      hi = -INFINITY;
      for (int b = first + t; b < last; b += kSelThreads) {
        if (bin_of(score[b]) == pivot) {
          lo = fminf(lo, score[b]);
          hi = fmaxf(hi, score[b]);
        }
      }
      lo = wg_reduce(lo, minf, smf) - err2;
      hi = wg_reduce(hi, maxf, smf) + err2;
      // certain ones, and those between
      int in = 0;
      for (int b = first + t; b < last; b += kSelThreads) {
        const float s = score[b];
        if (s > hi) {
          choose(b);
          ++in;
        } else if (s >= lo) {
          const int k = atomicAdd(&num_cand, 1);
          if (k < kCand) cand_at[k] = b;
        }
      }
      in = wg_reduce(in, addi, smi);
      const int left = want - in, cands = num_cand;
      slow = cands > kCand;
      if (!slow && cands == left) {
        for (int k = t; k < cands; k += kSelThreads) choose(cand_at[k]);
      } else if (!slow) {
        for (int k = w; k < cands; k += kSelWaves) {
          const uint64_t key = exact_key<D>(a, q, g, table, kvh, cand_at[k]);
          if (lane == 0) cand_key[k] = key;
        }
        __syncthreads();
        for (int k = t; k < cands; k += kSelThreads) {
          int before = 0;
          for (int j = 0; j < cands; ++j)
            before += cand_key[j] > cand_key[k] ||
                      (cand_key[j] == cand_key[k] && cand_at[j] < cand_at[k]);
          if (before < left) choose(cand_at[k]);
        }
      }
    }
    if (slow) {
      // many blocks at the border (equal ones), or scores that are not finite: every key in 64
      // bits, in the workspace's two halves, and a search for the last chosen key bit by bit
      uint32_t* kh = reinterpret_cast<uint32_t*>(score);
      uint32_t* kl = reinterpret_cast<uint32_t*>(low);
      const bool all = !(isfinite(err2) && isfinite(mn) && isfinite(mx) && isfinite(range));
      for (int b0 = first + w * 64; b0 < last; b0 += kSelThreads) {
        const int b = b0 + lane;
        const float s = b < last ? score[b] : 0.f;
        uint64_t key = !all && s > hi ? ~0ull : 0ull;
        uint64_t todo = __builtin_amdgcn_ballot_w64(b < last && (all || (s >= lo && s <= hi)));
        while (todo != 0) {
          const int k = __builtin_ctzll(todo);
          todo &= todo - 1;
          const uint64_t x = exact_key<D>(a, q, g, table, kvh, b0 + k);
          if (lane == k) key = x;
        }
        if (b < last) {
          kh[b] = (uint32_t)(key >> 32);
          kl[b] = (uint32_t)key;
        }
      }
      __syncthreads();
      auto key_at = [&](int b) { return (uint64_t)kh[b] << 32 | kl[b]; };
      uint64_t cut = 0;  // the largest key that at least `want` blocks reach
      for (int bit = 63; bit >= 0; --bit) {
        const uint64_t probe = cut | 1ull << bit;
        int c = 0;
        for (int b = first + t; b < last; b += kSelThreads) c += key_at(b) >= probe;
        if (wg_reduce(c, addi, smi) >= want) cut = probe;
      }
      int c = 0;
      for (int b = first + t; b < last; b += kSelThreads) {
        if (key_at(b) > cut) {
          choose(b);
          ++c;
        }
      }
      c = wg_reduce(c, addi, smi);
      if (w == 0) {  // the rest from the equal ones, lowest index first
        int left = want - c;
        for (int b0 = first; b0 < last && left > 0; b0 += 64) {
          const int b = b0 + lane;
          const bool eq = b < last && key_at(b) == cut;
          const uint64_t m = __builtin_amdgcn_ballot_w64(eq);
          if (eq && __builtin_popcountll(m & ((1ull << lane) - 1)) < left) choose(b);
          left -= __builtin_popcountll(m);
        }
      }
    }
  }
  __syncthreads();
  // the chosen ones in ascending order
  int before = 0;
  for (int k0 = 0; k0 < (n + 31) / 32; k0 += kSelThreads) {
    const int k = k0 + t;
    uint32_t bits = k < (n + 31) / 32 ? chosen[k] : 0u;
    const int mine = __builtin_popcount(bits);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(incl, o);
      if (lane >= o) incl += u;
    }
    __syncthreads();
    if (lane == 63) smi[w] = incl;
    __syncthreads();
    int at = before + incl - mine;
    for (int j = 0; j < kSelWaves; ++j) {
      if (j < w) at += smi[j];
      before += smi[j];
    }
    while (bits != 0u) {
      sel[at++] = k * 32 + __builtin_ctz(bits);
      bits &= bits - 1u;
    }
  }
}

}  // namespace

size_t select_workspace_bytes(int64_t items, int32_t max_len, int32_t blocks) {
  const int64_t n = ((int64_t)max_len + kBlockSize - 1) / kBlockSize;
  if (n <= blocks) return 0;  // every block is chosen
  const int64_t stride = (n + 15) / 16 * 16;
  return (size_t)(items * (2 * stride + stride / 16)) * sizeof(float);
}

hipError_t launch_select_blocks(SelectArgs a, int head_dim, void* workspace, hipStream_t stream) {
  const int64_t items = a.rows * a.hkv;
  const int64_t n = std::min<int64_t>(((int64_t)a.max_len + kBlockSize - 1) / kBlockSize, a.max_blocks);
  a.stride = (((int64_t)a.max_len + kBlockSize - 1) / kBlockSize + 15) / 16 * 16;
  a.scores = static_cast<float*>(workspace);
  a.low = a.scores + items * a.stride;
  a.tile_most = a.low + items * a.stride;
  const bool wide = head_dim == 128;
  if (n > a.blocks && a.blocks > a.sink + a.recent) {
    const int64_t chunks = (n + 16 * kScoreWaves - 1) / (16 * kScoreWaves);
    const int64_t total = items * chunks;
    hipLaunchKernelGGL(wide ? score_kernel<128> : score_kernel<64>,
                       dim3((unsigned)std::min<int64_t>(total, 1 << 20)), dim3(64 * kScoreWaves), 0,
                       stream, a, (int)chunks, total);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  hipLaunchKernelGGL(wide ? select_kernel<128> : select_kernel<64>, dim3((unsigned)items),
                     dim3(kSelThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace pkv
