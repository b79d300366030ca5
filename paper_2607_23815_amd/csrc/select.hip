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
// One wave takes several tiles of 16 blocks of one row with the next tile's loads in flight. Rows of
// longer suffixes share their sequence's bounds: a wave then keeps 48 or 64 blocks' bounds in registers
// and runs the rows of 64 through them, as many rows a product as its 16 lines hold heads.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "device_utils.h"
#include "launch.h"
#include "wave_utils.h"

namespace pkv {
namespace {

constexpr int kScoreWaves = 4;
constexpr int kTileBlocks = 16;      // blocks of a product
constexpr int kMaxTiles = 3;         // tiles of one row that a wave takes at most
template <int D>
constexpr int kHeldTiles = D == 128 ? 3 : 4;  // tiles that a wave holds for a group of rows

// The row's blocks (those with a visible key), as both kernels count them.
__device__ __forceinline__ int row_blocks(const SelectArgs& a, int64_t row) {
  const int len = min(a.row_lens[row], a.max_len);
  return len <= 0 ? 0 : min((len - 1) / kBlockSize + 1, a.max_blocks);
}
__device__ __forceinline__ int row_sequence(const SelectArgs& a, int64_t row) {
  const int s = a.row_seq != nullptr ? a.row_seq[row] : (int)row;
  return s >= 0 && s < a.num_seqs ? s : -1;
}

// The parts of two bf16 with the sign bit `side`, zeros in the others' place.
__device__ __forceinline__ uint32_t one_side(uint32_t w, int side) {
  typedef __attribute__((ext_vector_type(2))) int16_t s16x2;
  const uint32_t neg = __builtin_bit_cast(uint32_t, (s16x2)(__builtin_bit_cast(s16x2, w) >> 15));
  return side ? w & neg : w & ~neg;
}
// The larger |bf16| of each half of two words, as bits.
__device__ __forceinline__ uint32_t most_of(uint32_t most, uint32_t w) {
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
  return __builtin_bit_cast(uint32_t,
                            __builtin_elementwise_max(__builtin_bit_cast(u16x2, most),
                                                      __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
}
// Over the wave, a NaN as infinity: a maximum of floats would pass a NaN over, and with it all that it
// stands for.
__device__ __forceinline__ float most_value(uint32_t most) {
  return __uint_as_float(min(wave_all(max(most & 0xFFFFu, most >> 16), Max()), 0x7F80u) << 16);
}
// The largest of n of a lane's four sums; +infinity if one of them (or their sum) is not finite.
template <int n>
__device__ __forceinline__ float best_of(const f32x4& s, int e) {
  float best = s[e], sum = s[e];
#pragma unroll
  for (int k = 1; k < n; ++k) {
    best = fmaxf(best, s[e + k]);
    sum += s[e + k];
  }
  return fabsf(sum) < INFINITY ? best : INFINITY;
}

template <int D>
struct Box {  // 16 blocks' bounds: lane (block col, chunk group grp)
  u32x4 v[2][D / 32];
};
template <int D>
__device__ __forceinline__ void load_box(const SelectArgs& a, Box<D>& x, int id, int kvh) {
  const int grp = (threadIdx.x & 63) >> 4;
  if (id < 0 || id >= a.num_blocks) id = 0;
  const uint16_t* box = a.bounds + ((size_t)id * a.hkv + kvh) * 2 * D + grp * 8;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) x.v[side][kk] = ld16(box + side * D + kk * 32);
  }
}
template <int D>
__device__ __forceinline__ uint32_t box_most(const Box<D>& x) {
  uint32_t most = 0u;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
#pragma unroll
      for (int e = 0; e < 4; ++e) most = most_of(most, x.v[side][kk][e]);
    }
  }
  return most;
}
// q (16 heads x D, lane (head col, chunk group)) split into its positive and negative parts.
template <int D>
struct Sides {
  u32x4 v[2][D / 32];
};
template <int D>
__device__ __forceinline__ void split_q(const u32x4 (&q)[D / 32], Sides<D>& x) {
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x.v[side][kk][e] = one_side(q[kk][e], side);
    }
  }
}
// Lane (block col, group grp) receives the sums of heads 4 grp + 0..3.
template <int D>
__device__ __forceinline__ f32x4 score(const Sides<D>& q, const Box<D>& b) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk)
      s = mfma16(as_bf16x8(q.v[side][kk]), as_bf16x8(b.v[side][kk]), s);
  }
  return s;
}

// The group's heads as a product's lines (those past the group's hold its last one again: no new
// maximum).
template <int D>
__device__ __forceinline__ void load_heads(const uint16_t* q, int g, u32x4 (&qv)[D / 32]) {
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) qv[kk] = ld16(q + min(col, g - 1) * D + kk * 32 + grp * 8);
}
// The scores of a tile's blocks, block col's in lane (col, any grp).
template <int D>
__device__ __forceinline__ float tile_scores(const Sides<D>& q, const Box<D>& b) {
  float best = best_of<4>(score<D>(q, b), 0);
  u32x2 x = with_row(__float_as_uint(best));
  best = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  x = with_half(__float_as_uint(best));
  return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}

// A wave per (row, run of tiles, kv head); a block's bounds of all heads lie together.
template <int D>
__global__ __launch_bounds__(64 * kScoreWaves) void score_row_kernel(const SelectArgs a, int runs,
                                                                     int tiles, int64_t total) {
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t work = (int64_t)blockIdx.x * kScoreWaves + wave; work < total;
       work += (int64_t)gridDim.x * kScoreWaves) {
    const int kvh = (int)(work % a.hkv);
    const int64_t row = work / a.hkv / runs;
    const int64_t item = row * a.hkv + kvh;
    const int t0 = (int)(work / a.hkv % runs) * tiles;
    const int n = row_blocks(a, row), seq = row_sequence(a, row);
    if (seq < 0 || n <= a.blocks || t0 * kTileBlocks >= n) continue;
    const int t1 = min(t0 + tiles, (n + kTileBlocks - 1) / kTileBlocks);
    const int32_t* table = a.tables + (size_t)seq * a.max_blocks;
    // the ids of the run's blocks
    static_assert(kMaxTiles * kTileBlocks <= 64, "one of each lane");
    const int ids = table[min(t0 * kTileBlocks + lane, n - 1)];
    const int g = a.hq / a.hkv;
    u32x4 qv[D / 32];
    load_heads<D>(a.q + ((size_t)row * a.hq + kvh * g) * D, g, qv);
    auto id_of = [=](int j) {  // of block col of the run's tile j
      return __builtin_amdgcn_ds_bpermute((j * kTileBlocks + col) * 4, ids);
    };
    Sides<D> q;
    Box<D> box[2];
    load_box<D>(a, box[0], id_of(0), kvh);
    split_q<D>(qv, q);
    float* out = a.scores + item * a.stride;
    float* most = a.tile_most + item * (a.stride / kTileBlocks);
    auto finish = [&](const Box<D>& b, int t) {
      const float best = tile_scores<D>(q, b);
      const float top = most_value(box_most<D>(b));
      if (grp == 0 && t * kTileBlocks + col < n) out[t * kTileBlocks + col] = best;
      if (lane == 0) most[t] = top;
    };
    for (int t = t0; t < t1; t += 2) {
      if (t + 1 < t1) load_box<D>(a, box[1], id_of(t + 1 - t0), kvh);
      finish(box[0], t);
      if (t + 1 >= t1) break;
      if (t + 2 < t1) load_box<D>(a, box[0], id_of(t + 2 - t0), kvh);
      finish(box[1], t + 1);
    }
  }
}

// Rows of a group: 64 at most, and as many as 64 KB of LDS hold of their heads' queries.
template <int D, int kHeads>
constexpr int kGroupTiles = std::min(64 * kHeads / kTileBlocks, 2048 / D);

// A workgroup per (group of rows, kv head, held tiles of its waves). The queries of the group's rows go
// to LDS in operand order, kTileBlocks / kHeads rows a product (kHeads: the group's heads rounded up
// to a power of two). Each wave holds the bounds of its blocks in registers, one run of rows of one
// sequence after the other, and takes the queries through them.
template <int D, int kHeads>
__global__ __launch_bounds__(64 * kScoreWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void score_rows_kernel(const SelectArgs a, int chunks, int group, int64_t total) {
  constexpr int kRows = kTileBlocks / kHeads;  // rows of a product
  constexpr int KK = D / 32;
  constexpr int kHeld = kHeldTiles<D>;
  __shared__ __align__(16) u32x4 qs[kGroupTiles<D, kHeads>][KK][64];
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = a.hq / a.hkv;
  for (int64_t work = blockIdx.x; work < total; work += gridDim.x) {
    const int b0 = ((int)(work % chunks) * kScoreWaves + wave) * kTileBlocks * kHeld;
    const int kvh = (int)(work / chunks % a.hkv);
    const int64_t row0 = work / chunks / a.hkv * group;
    // lane i: row i of the group, its sequence and the blocks to score (0: none)
    const int64_t mine = row0 + lane;
    const int seq = lane < group && mine < a.rows ? row_sequence(a, mine) : -1;
    int n = seq >= 0 ? row_blocks(a, mine) : 0;
    // a product's line: head col % kHeads of row col / kHeads (past the group's heads its last one
    // again: no new maximum)
    const int head = min(col % kHeads, g - 1);
    __syncthreads();  // (the readers of the loop's last pass)
    constexpr int kMineTiles = (kGroupTiles<D, kHeads> + kScoreWaves - 1) / kScoreWaves;
    u32x4 qv[kMineTiles][KK];  // (every load before the first is waited for; rows past the last: its)
#pragma unroll
    for (int k = 0; k < kMineTiles; ++k) {
      const int64_t row = min(row0 + (wave + k * kScoreWaves) * kRows + col / kHeads, a.rows - 1);
      const uint16_t* from = a.q + ((size_t)row * a.hq + kvh * g + head) * D + grp * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        if ((wave + k * kScoreWaves) * kRows < group) qv[k][kk] = ld16(from + kk * 32);
    }
    if (n <= a.blocks || n <= b0) n = 0;
    uint64_t todo = __builtin_amdgcn_ballot_w64(n > 0);
#pragma unroll
    for (int k = 0; k < kMineTiles; ++k) {
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        if ((wave + k * kScoreWaves) * kRows < group) qs[wave + k * kScoreWaves][kk][lane] = qv[k][kk];
    }
    __syncthreads();
    while (todo != 0) {
      const int first = __builtin_ctzll(todo);
      const int s = __builtin_amdgcn_readlane(seq, first);
      const uint64_t same = __builtin_amdgcn_ballot_w64(seq == s) >> first;
      const int end = first + (~same == 0 ? 64 : __builtin_ctzll(~same));  // (past the run)
      const int most_n = wave_all(lane >= first && lane < end ? n : 0, Max());
      todo &= end >= 64 ? 0 : ~0ull << end;
      Box<D> box[kHeld];
      const int id = a.tables[(size_t)s * a.max_blocks + min(b0 + lane, most_n - 1)];
#pragma unroll
      for (int j = 0; j < kHeld; ++j)  // (column col holds neighbours, which are stored together)
        load_box<D>(a, box[j], __builtin_amdgcn_ds_bpermute((col * kHeld + j) * 4, id), kvh);
      uint32_t most = 0u;
#pragma unroll
      for (int j = 0; j < kHeld; ++j) most = most_of(most, box_most<D>(box[j]));
      const float top = most_value(most);
      constexpr int kMine = kHeads >= 4 ? 1 : 4 / kHeads;  // rows of a lane
      const bool writer = kHeads <= 4 || 4 * grp % kHeads == 0;
      for (int t = first / kRows; t * kRows < end; ++t) {
        u32x4 qv[KK];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) qv[kk] = qs[t][kk][lane];
        Sides<D> q;
        split_q<D>(qv, q);
        // the lane's rows: blocks to score from this lane's block on, and where they go
        int left[kMine];
        int64_t to[kMine];
#pragma unroll
        for (int e = 0; e < kMine; ++e) {
          const int at = t * kRows + (kHeads >= 4 ? 4 * grp / kHeads : kMine * grp + e);
          const int rn = __builtin_amdgcn_ds_bpermute(at * 4, n);
          left[e] = writer && at >= first && at < end ? rn - b0 - col * kHeld : 0;
          to[e] = ((row0 + at) * a.hkv + kvh) * a.stride + b0;
        }
        // (every tile's products before the first result is looked at)
        f32x4 sc[kHeld];
#pragma unroll
        for (int j = 0; j < kHeld; ++j) sc[j] = score<D>(q, box[j]);
        float best[kHeld][kMine];
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
#pragma unroll
          for (int e = 0; e < kMine; ++e) best[j][e] = best_of<4 / kMine>(sc[j], e * (4 / kMine));
          if constexpr (kHeads >= 8) {
            const u32x2 x = with_row(__float_as_uint(best[j][0]));
            best[j][0] = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
          }
          if constexpr (kHeads == 16) {
            const u32x2 x = with_half(__float_as_uint(best[j][0]));
            best[j][0] = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
          }
        }
#pragma unroll
        for (int e = 0; e < kMine; ++e) {
          if (left[e] <= 0) continue;
          float* dst = a.scores + to[e] + col * kHeld;  // (the row's stride holds whole chunks)
#pragma unroll
          for (int j = 0; j < kHeld; ++j) dst[j] = best[j][e];
          if (col == 0) a.tile_most[to[e] / kTileBlocks] = top;
        }
      }
    }
  }
}

__device__ __forceinline__ double row_sum(double x) {  // over 16 lanes (lane 0's order counts)
  auto step = [&](auto ror) {
    constexpr int kCtrl = decltype(ror)::value;
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    x += __longlong_as_double((long long)((uint64_t)dpp<kCtrl>((uint32_t)(u >> 32)) << 32 |
                                          dpp<kCtrl>((uint32_t)u)));
  };
  step(std::integral_constant<int, 0x128>());
  step(std::integral_constant<int, 0x124>());
  step(std::integral_constant<int, 0x122>());
  step(std::integral_constant<int, 0x121>());
  return x;
}

// Scores in 64 bits by one wave, four blocks at a time: 16 lanes take block b, each of them D / 16
// dims for every head. The key's unsigned order is the scores' order (a bound or query that is
// not finite makes it +infinity); it is never 0 and never ~0, and valid in the first of the 16 lanes.
template <int D>
__device__ __forceinline__ uint64_t exact_key(const SelectArgs& a, const uint16_t* q, int g,
                                              const int32_t* table, int kvh, int b) {
  constexpr int PER = D / 16;
  const int lane = threadIdx.x & 63, part = lane & 15;
  int id = table[b];
  if (id < 0 || id >= a.num_blocks) id = 0;
  const uint16_t* box = a.bounds + ((size_t)id * a.hkv + kvh) * 2 * D + part * PER;
  uint16_t hb[PER], lb[PER];
  __builtin_memcpy(hb, __builtin_assume_aligned(box, 2 * PER), sizeof(hb));
  __builtin_memcpy(lb, __builtin_assume_aligned(box + D, 2 * PER), sizeof(lb));
  float hi[PER], lo[PER];
  bool odd = false;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    hi[e] = __uint_as_float((uint32_t)hb[e] << 16);
    lo[e] = __uint_as_float((uint32_t)lb[e] << 16);
    odd |= !isfinite(hi[e]) || !isfinite(lo[e]);
  }
  double best = -INFINITY;
  constexpr int kHeads = 256 / D;  // heads whose loads and sums run side by side
  for (int h0 = 0; h0 < g; h0 += kHeads) {
    uint16_t qb[kHeads][PER];
#pragma unroll
    for (int k = 0; k < kHeads; ++k)
      __builtin_memcpy(qb[k], __builtin_assume_aligned(q + min(h0 + k, g - 1) * D + part * PER, 2 * PER),
                       sizeof(qb[k]));
    double s[kHeads] = {};
#pragma unroll
    for (int e = 0; e < PER; ++e) {
#pragma unroll
      for (int k = 0; k < kHeads; ++k) {
        const float x = __uint_as_float((uint32_t)qb[k][e] << 16);
        odd |= !isfinite(x);
        s[k] = fma((double)x, (double)(x > 0.f ? hi[e] : lo[e]), s[k]);  // (the product is exact)
      }
    }
#pragma unroll
    for (int k = 0; k < kHeads; ++k) best = fmax(best, row_sum(s[k]));
  }
  const uint64_t odds = __builtin_amdgcn_ballot_w64(odd) >> (lane & 48) & 0xFFFFu;
  if (odds != 0) best = INFINITY;
  best += 0.;  // (-0 becomes +0: equal scores, equal keys)
  const uint64_t u = (uint64_t)__double_as_longlong(best);
  return u >> 63 ? ~u : u | 1ull << 63;
}

// Several 32-bit values combined over the workgroup at once.
template <int kThreads, int n, typename T, typename F>
__device__ __forceinline__ void wg_all(T (&v)[n], F op, T (*sm)[n]) {
  constexpr int kWaves = kThreads / 64;
#pragma unroll
  for (int k = 0; k < n; ++k) v[k] = wave_all(v[k], op);
  if constexpr (kWaves > 1) {
    __syncthreads();  // (sm's readers of the last call)
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < n; ++k) sm[threadIdx.x >> 6][k] = v[k];
    }
    __syncthreads();
    // (every lane of a row of 16 reads one wave's values; the waves divide the row evenly)
    static_assert(kWaves <= 16 && 16 % kWaves == 0, "waves fit a row of lanes");
#pragma unroll
    for (int k = 0; k < n; ++k) {
      T x = sm[threadIdx.x % kWaves][k];
      auto step = [&](uint32_t other) { x = op(x, __builtin_bit_cast(T, other)); };
      if constexpr (kWaves > 8) step(dpp<0x128>(__builtin_bit_cast(uint32_t, x)));
      if constexpr (kWaves > 4) step(dpp<0x124>(__builtin_bit_cast(uint32_t, x)));
      step(dpp<0x122>(__builtin_bit_cast(uint32_t, x)));
      step(dpp<0x121>(__builtin_bit_cast(uint32_t, x)));
      v[k] = x;
    }
  }
}
// The sum over the threads before this one, and over all.
template <int kThreads>
__device__ __forceinline__ int wg_before(int v, int* total, int* sm) {
  constexpr int kWaves = kThreads / 64;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int incl = wave_scan(v);
  __syncthreads();
  if (lane == 63) sm[w] = incl;
  __syncthreads();
  const int from = lane & 15;  // lane's wave
  const int sum = from < kWaves ? sm[from] : 0;
  *total = row_all(sum, Add());
  return incl - v + row_all(from < w ? sum : 0, Add());
}

// One workgroup per (row, kv head). Its scores stay in registers, 64 consecutive blocks per wave and
// register, at most kThreads * kEach (kEach 0: in memory, any number). kOwn: it takes the scores itself,
// where the other form reads those of a launch before.
template <int D, int kThreads, int kEach, bool kOwn = false>
__global__ __launch_bounds__(kThreads) void select_kernel(const SelectArgs a) {
  constexpr int kWaves = kThreads / 64;
  constexpr int kPer = kThreads == 1024 ? 2 : 8;  // bins of a thread
  constexpr int kBins = kPer * kThreads;
  constexpr int kCand = kThreads == 64 ? 128 : 512;  // blocks near the border that are ranked in LDS
  constexpr int kWords = (kEach > 0 ? kThreads * kEach : kSelectMaxBlocks + kThreads) / 64;
  __shared__ uint64_t chosen[kWords];  // a bit per block from `first` on, a word per wave and chunk
  __shared__ __align__(16) uint32_t bins[kBins];
  __shared__ __align__(16) uint16_t heads[16 * D];  // the group's queries
  __shared__ uint64_t cand_key[kCand];
  __shared__ int cand_at[kCand];
  __shared__ float sm5[kWaves][5];
  __shared__ int sm1[kWaves][1], sms[kWaves];
  __shared__ int num_cand, pivot;
  __shared__ float own[kOwn ? kThreads * kEach : 1];
  const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t item = blockIdx.x;
  const int64_t row = item / a.hkv;
  const int kvh = (int)(item % a.hkv);
  const int seq = row_sequence(a, row);
  if (seq < 0) return;  // a padding row
  const int n = row_blocks(a, row);
  int32_t* sel = a.sel + item * a.blocks;
  if (n <= a.blocks) {  // every block
    for (int k = t; k < a.blocks; k += kThreads) sel[k] = k < n ? k : -1;
    return;
  }
  const int first = a.sink, last = n - a.recent;  // [first, last) goes by score
  const int want = a.blocks - a.sink - a.recent;
  for (int k = t; k < a.sink + a.recent; k += kThreads) {
    if (k < a.sink) sel[k] = k;
    else sel[want + k] = last + (k - a.sink);
  }
  if (want == 0) return;
  float* scores = a.scores + item * a.stride;
  float* low = a.low + item * a.stride;
  const int32_t* table = a.tables + (size_t)seq * a.max_blocks;
  const int g = a.hq / a.hkv;
  const uint16_t* q = a.q + ((size_t)row * a.hq + kvh * g) * D;
  uint32_t most = 0u;
  if constexpr (kOwn) {  // tiles of 16 blocks in turn for the waves, two of a wave's in flight
    const int col = lane & 15, grp = lane >> 4, tiles = (n + kTileBlocks - 1) / kTileBlocks;
    u32x4 qv[D / 32];
    load_heads<D>(q, g, qv);
    Sides<D> sides;
    for (int t0 = w; t0 < tiles; t0 += 2 * kWaves) {
      const int t1 = t0 + kWaves;
      Box<D> box[2];
      const int id0 = table[min(t0 * kTileBlocks + col, n - 1)];
      const int id1 = table[min(t1 * kTileBlocks + col, n - 1)];  // (past the last tile its block again)
      load_box<D>(a, box[0], id0, kvh);
      load_box<D>(a, box[1], id1, kvh);
      if (t0 == w) split_q<D>(qv, sides);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int b = (k == 0 ? t0 : t1) * kTileBlocks + col;
        const float best = tile_scores<D>(sides, box[k]);
        most = most_of(most, box_most<D>(box[k]));
        if (grp == 0 && b < n) own[b] = best;
      }
    }
    __syncthreads();
  }
  auto score_of = [&](int b) { return kOwn ? own[b] : scores[b]; };

  // the wave's blocks: `chunks` times 64 from `base` on; a place past the last holds a NaN, which no
  // comparison, minimum or maximum below takes up
  const int chunks = ((last - first + 63) / 64 + kWaves - 1) / kWaves;
  const int base = first + w * chunks * 64;
  float s[kEach > 0 ? kEach : 1];
  auto block_of = [&](int k) { return base + 64 * k + lane; };
  auto value = [&](int b) {
    const float x = score_of(min(b, last - 1));
    return b < last ? x : NAN;
  };
  if constexpr (kOwn) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) s[k] = k < chunks ? value(block_of(k)) : NAN;
  } else if constexpr (kEach > 0) {
    // (every load before the first use, and none in a branch; past the last score they read zeros)
#pragma unroll
    for (int k = 0; k < kEach; ++k) s[k] = __uint_as_float(buf_ld4(scores, last * 4, block_of(k) * 4));
#pragma unroll
    for (int k = 0; k < kEach; ++k) s[k] = k < chunks && block_of(k) < last ? s[k] : NAN;
  }
  auto each = [&](auto f) {  // f(block, score), chunk by chunk
    if constexpr (kEach > 0) {
#pragma unroll
      for (int k = 0; k < kEach; ++k)
        if (k < chunks) f(block_of(k), s[k]);
    } else {
      for (int k = 0; k < chunks; ++k) f(block_of(k), value(block_of(k)));
    }
  };
  if (t == 0) num_cand = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) bins[t * kPer + k] = 0u;
  auto choose = [&](int b) {
    const int at = b - first;
    atomicOr(reinterpret_cast<uint32_t*>(chosen) + (at >> 5), 1u << (at & 31));
  };

  // the error of a 32-bit score: 2 D products summed in some order, each addition off by at most
  // 2^-23 of the sum of their magnitudes, |q|_1 max |bound|; tiny values may count as zeros
  float all[5] = {0.f, 0.f, 0.f, -INFINITY, -INFINITY};  // |q|_1, max |q|, max |bound|, -min s, max s
  for (int h0 = 4 * w; h0 < g; h0 += 4 * kWaves) {  // (16 lanes a head)
    const int at = min(h0 + (lane >> 4), g - 1) * D + (lane & 15) * (D / 16);
    uint16_t part[D / 16];
    __builtin_memcpy(part, __builtin_assume_aligned(q + at, D / 8), sizeof(part));
    __builtin_memcpy(__builtin_assume_aligned(&heads[at], D / 8), part, sizeof(part));
    float norm = 0.f;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      const float x = fabsf(__uint_as_float((uint32_t)part[e] << 16));
      norm += x;
      all[1] = fmaxf(all[1], x);
    }
    all[0] = fmaxf(all[0], row_all(norm, Add()));
  }
  if constexpr (kOwn) all[2] = most_value(most);
  else for (int k = t; k * a.most_step * kTileBlocks < n; k += kThreads)
    all[2] = fmaxf(all[2], a.tile_most[item * (a.stride / kTileBlocks) + k * a.most_step]);
  each([&](int, float x) {
    all[3] = fmaxf(all[3], -x);
    all[4] = fmaxf(all[4], x);
  });
  wg_all<kThreads>(all, Max(), sm5);
  const float tiny = 0x1p-118f;
  const float err2 = 2.f * (0x1p-15f * 1.01f * all[0] * all[2] + tiny * (1.f + all[1] + all[2]));
  const float mn = -all[3], range = all[4] + all[3];
  const bool odd = !(isfinite(err2) && isfinite(all[4]) && isfinite(mn) && isfinite(range));

  // how the scores spread: a histogram between the least and the largest finds the bin of the last
  // chosen one (places past the last count into bin 0, which nothing looks past)
  bool slow = odd;
  const float per = range > 0.f ? (kBins - 1) / range : 0.f;
  auto bin_of = [&](float x) {  // (a NaN's is 0)
    return (int)fminf(fmaxf((x - mn) * per, 0.f), kBins - 1.f);
  };
  float lo = 0.f, hi = 0.f;
  __syncthreads();
  if (!slow) {
    each([&](int, float x) { atomicAdd(&bins[bin_of(x)], 1u); });
    __syncthreads();
    // thread t counts bins [kPer (kThreads - 1 - t), + kPer): from the top
    uint32_t mine[kPer];
    __builtin_memcpy(mine, __builtin_assume_aligned(&bins[(kThreads - 1 - t) * kPer], 4 * kPer),
                     sizeof(mine));
    int sum = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) sum += mine[k];
    int total;
    const int before = wg_before<kThreads>(sum, &total, sms);
    if (before < want && want <= before + sum) {  // (one thread)
      int above = before;
#pragma unroll
      for (int k = kPer - 1; k >= 0; --k) {
        if (above < want && want <= above + (int)mine[k]) pivot = (kThreads - 1 - t) * kPer + k;
        above += mine[k];
      }
    }
    __syncthreads();
    // Fewer than `want` scores lie above that bin, at least as many from its lower edge on. A score's
    // place, (x - mn) * per, is off by less than 2^-22 of itself: 2^-20 of the range covers the edges.
    const float width = range / (kBins - 1), slack = range * 0x1p-20f;
    lo = mn + pivot * width - slack - err2;
    hi = mn + (pivot + 1) * width + slack + err2;
    // certain ones, and those between
    int sure = 0;
    each([&](int b, float x) {
      const uint64_t m = __builtin_amdgcn_ballot_w64(x > hi);
      sure += __builtin_popcountll(m);
      if (lane == 0) chosen[(b - first) >> 6] = m;  // (its lane's block is the chunk's first)
      if (x >= lo && x <= hi) {
        const int k = atomicAdd(&num_cand, 1);
        if (k < kCand) cand_at[k] = b;
      }
    });
    int in[1] = {lane == 0 ? sure : 0};
    wg_all<kThreads>(in, Add(), sm1);
    __syncthreads();  // (a single wave's candidates too)
    const int left = want - in[0], cands = num_cand;
    slow = cands > kCand;
    if (!slow && cands == left) {
      for (int k = t; k < cands; k += kThreads) choose(cand_at[k]);
    } else if (!slow) {
      for (int k0 = 4 * w; k0 < cands; k0 += 4 * kWaves) {
        const int k = k0 + (lane >> 4);
        const uint64_t key = exact_key<D>(a, heads, g, table, kvh, cand_at[min(k, cands - 1)]);
        if (k < cands && (lane & 15) == 0) cand_key[k] = key;
      }
      __syncthreads();
      for (int k = t; k < cands; k += kThreads) {
        int ahead = 0;
        for (int j = 0; j < cands; ++j)
          ahead += cand_key[j] > cand_key[k] ||
                   (cand_key[j] == cand_key[k] && cand_at[j] < cand_at[k]);
        if (ahead < left) choose(cand_at[k]);
      }
    }
  }
  if (slow) {
    // many blocks at the border (equal ones), or scores that are not finite: every key in 64
    // bits, in the workspace's two halves, and a search for the last chosen key bit by bit
    uint32_t* kh = reinterpret_cast<uint32_t*>(scores);
    uint32_t* kl = reinterpret_cast<uint32_t*>(low);
    for (int b0 = first + w * 64; b0 < last; b0 += kThreads) {
      const int b = b0 + lane;
      const float x = b < last ? score_of(b) : 0.f;
      uint64_t key = !odd && x > hi ? ~0ull : 0ull;
      const uint64_t todo = __builtin_amdgcn_ballot_w64(b < last && (odd || (x >= lo && x <= hi)));
      for (int k = 0; k < 64; k += 4) {
        if ((todo >> k & 15) == 0) continue;
        const int at = k + (lane >> 4);  // block b0 + at, by the lane's 16
        const uint64_t exact = exact_key<D>(a, heads, g, table, kvh, min(b0 + at, last - 1));
        const int from = (lane & 3) * 16 * 4;  // (to lane k + j from lane 16 j)
        const uint32_t eh = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(exact >> 32));
        const uint32_t el = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(uint32_t)exact);
        if ((lane & ~3) == k && (todo >> lane & 1)) key = (uint64_t)eh << 32 | el;
      }
      if (b < last) {
        kh[b] = (uint32_t)(key >> 32);
        kl[b] = (uint32_t)key;
      }
    }
    __syncthreads();
    for (int k = t; k < kWaves * chunks; k += kThreads) chosen[k] = 0;
    auto key_at = [&](int b) { return (uint64_t)kh[b] << 32 | kl[b]; };
    uint64_t cut = 0;  // the largest key that at least `want` blocks reach
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t probe = cut | 1ull << bit;
      int c[1] = {0};
      for (int b = first + t; b < last; b += kThreads) c[0] += key_at(b) >= probe;
      wg_all<kThreads>(c, Add(), sm1);
      if (c[0] >= want) cut = probe;
    }
    int c[1] = {0};
    for (int b = first + t; b < last; b += kThreads) {
      if (key_at(b) > cut) {
        choose(b);
        ++c[0];
      }
    }
    wg_all<kThreads>(c, Add(), sm1);
    if (w == 0) {  // the rest from the equal ones, lowest index first
      int left = want - c[0];
      for (int b0 = first; b0 < last && left > 0; b0 += 64) {
        const int b = b0 + lane;
        const bool eq = b < last && key_at(b) == cut;
        const uint64_t m = __builtin_amdgcn_ballot_w64(eq);
        if (eq && __builtin_popcountll(m & ((1ull << lane) - 1)) < left) choose(b);
        left -= __builtin_popcountll(m);
      }
    }
  }
  __syncthreads();
  // the chosen ones in ascending order: every wave counts the words' bits, 64 words at a time, and
  // writes out its part of the words
  int at = a.sink;
  for (int k0 = 0; k0 < kWaves * chunks; k0 += 64) {
    const uint64_t word = k0 + lane < kWaves * chunks ? chosen[k0 + lane] : 0;
    const int bits = __builtin_popcountll(word), upto = wave_scan(bits);
    const int end = min(64, kWaves * chunks - k0);
    for (int k = w; k < end; k += kWaves) {
      const uint64_t m = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(word >> 32), k) << 32 |
                         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)word, k);
      const int from = at + __builtin_amdgcn_readlane(upto - bits, k);
      if (m >> lane & 1)
        sel[from + __builtin_popcountll(m & ((1ull << lane) - 1))] = first + (k0 + k) * 64 + lane;
    }
    at += __builtin_amdgcn_readlane(upto, 63);
  }
}

}  // namespace

// A row's scores in the workspace: whole chunks of both head dims' score_rows_kernel.
static int64_t select_stride(int64_t n) { return (n + 191) / 192 * 192; }

size_t select_workspace_bytes(int64_t items, int32_t max_len, int32_t blocks) {
  const int64_t n = ((int64_t)max_len + kBlockSize - 1) / kBlockSize;
  if (n <= blocks) return 0;  // every block is chosen
  const int64_t stride = select_stride(n);
  return (size_t)(items * (2 * stride + stride / kTileBlocks)) * sizeof(float);
}

namespace {

// Short rows take their scores in the workgroup that chooses: one launch, and no scores in memory. 8
// heads of 128 dims (us, so and as two launches): one sequence of up to 62 blocks 6.7 and 10.4, 512 30.2 and
// 41.5; one of 250 9.9 and 11.5, 64 17.1 and 21.9, 256 45.7 and 57.4; one of 500 12.1 and 11.0, 256 86.6 and
// 97.5. Rows that share a sequence read its bounds once a group in the other form: 1220 items of 62 blocks
// 9.4 and 11.8, 6100 20.8 and 20.6, but 1220 of 250 17.6 and 14.1; 120 of 250 8.1 and 11.0.
bool select_one_launch(const SelectArgs& a, int64_t items, int64_t n) {
  if (n > 512 || a.blocks == a.sink + a.recent) return false;
  return a.row_seq == nullptr || items <= 512 || (n <= 64 && items <= 4096);
}

template <int D>
hipError_t launch_scores(const SelectArgs& a, int64_t items, int64_t n, hipStream_t stream) {
  constexpr int64_t kMostWorkgroups = 1 << 20;  // (a launch's loop takes the others)
  const int64_t tiles = (n + kTileBlocks - 1) / kTileBlocks;
  if (a.row_seq == nullptr) {
    // Short runs of tiles: waves of a few microseconds keep a row's heads, whose bounds lie together in
    // memory, side by side in time. 256 sequences of 8-32k keys, 8 heads (us, both launches, at 1, 2, 3, 4,
    // 6, 8, 16 tiles): 336, 271, 261, 281, 264, 346, 350; with one head 66, 54, 49, 55, 51, 56, 56; 64 with
    // 8 heads 94, 79, 79, 85, 81, 94, 97; but 16 33.9, 31.1, 31.7, one of 120k 20.7, 20.2, 22.2.
    const int64_t run = items * tiles >= 32768 ? kMaxTiles : 2;
    const int64_t runs = (tiles + run - 1) / run, total = items * runs;
    const int64_t wgs = std::min((total + kScoreWaves - 1) / kScoreWaves, kMostWorkgroups);
    hipLaunchKernelGGL(score_row_kernel<D>, dim3((unsigned)wgs), dim3(64 * kScoreWaves), 0, stream,
                       a, (int)runs, (int)run, total);
    return hipGetLastError();
  }
  const int64_t chunks = (tiles + kHeldTiles<D> * kScoreWaves - 1) / (kHeldTiles<D> * kScoreWaves);
  const int g = a.hq / a.hkv;
  auto launch = [&](auto heads) {
    constexpr int kHeads = decltype(heads)::value;
    constexpr int kRows = kTileBlocks / kHeads;
    // Large groups read the bounds less often, small ones fill the chip where rows are few (305 rows, 4
    // heads, up to 5 chunks of blocks: 27.3 us at 64 rows a group, 21.5 halved to 256 workgroups).
    int group = kGroupTiles<D, kHeads> * kRows;
    int64_t total = 0;
    for (;; group /= 2) {
      total = (a.rows + group - 1) / group * a.hkv * chunks;
      if (group <= kRows || total >= kComputeUnits) break;
    }
    hipLaunchKernelGGL((score_rows_kernel<D, kHeads>),
                       dim3((unsigned)std::min(total, kMostWorkgroups)), dim3(64 * kScoreWaves), 0,
                       stream, a, (int)chunks, group, total);
  };
  if (g == 1) launch(std::integral_constant<int, 1>());
  else if (g == 2) launch(std::integral_constant<int, 2>());
  else if (g <= 4) launch(std::integral_constant<int, 4>());
  else if (g <= 8) launch(std::integral_constant<int, 8>());
  else launch(std::integral_constant<int, 16>());
  return hipGetLastError();
}

template <int D>
hipError_t launch_select(const SelectArgs& a, int64_t items, int64_t n, hipStream_t stream) {
  if (select_one_launch(a, items, n)) {  // (a wave alone has no barriers: up to 64 blocks, 30 us against 40)
    auto* kern = n <= 64 ? select_kernel<D, 64, 1, true> : select_kernel<D, 256, 2, true>;
    hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(n <= 64 ? 64 : 256), 0, stream, a);
    return hipGetLastError();
  }
  // Registers for the longest row the call can have. Short rows take a wave each where there are many:
  // no barriers, and more rows at once (6100 items of up to 1024 blocks 47.8 us with their scores
  // against 60.5 with four waves, 12200 of 128 dims 92.0 and 135.1; but 400 items 18.6 and 16.2).
  const bool t64 = n <= 1024 && items >= 1024;
  const int threads = t64 ? 64 : n <= 2048 ? 256 : 1024;
  auto* kern = t64   ? select_kernel<D, 64, 16>
               : n <= 2048 ? select_kernel<D, 256, 8>
               : n <= 8192 ? select_kernel<D, 1024, 8>
                           : select_kernel<D, 1024, 0>;
  hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(threads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_select_blocks(SelectArgs a, int head_dim, void* workspace, hipStream_t stream) {
  const int64_t items = a.rows * a.hkv;
  const int64_t most = ((int64_t)a.max_len + kBlockSize - 1) / kBlockSize;
  const int64_t n = std::min<int64_t>(most, a.max_blocks);
  a.stride = select_stride(most);
  a.most_step = a.row_seq == nullptr ? 1 : head_dim == 128 ? kHeldTiles<128> : kHeldTiles<64>;
  a.scores = static_cast<float*>(workspace);
  a.low = a.scores + items * a.stride;
  a.tile_most = a.low + items * a.stride;
  const bool wide = head_dim == 128;
  if (n > a.blocks && a.blocks > a.sink + a.recent && !select_one_launch(a, items, n)) {
    const hipError_t err = wide ? launch_scores<128>(a, items, n, stream)
                                : launch_scores<64>(a, items, n, stream);
    if (err != hipSuccess) return err;
  }
  return wide ? launch_select<128>(a, items, n, stream) : launch_select<64>(a, items, n, stream);
}

}  // namespace pkv
