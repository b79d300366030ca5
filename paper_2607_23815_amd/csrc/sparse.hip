// Attention over chosen blocks (gfx950): row t's g query heads of a kv head attend over the keys of
// the blocks that the row's list names for that kv head,
//   out[t][h] = sum_p softmax_p(scale <q[t][h], K[p]>) V[p],  p in the listed blocks, p < row_lens[t].
// The running maximum and weight sum of the softmax make it one pass over the keys. A wave takes
// four blocks at a time straight into the matrix-core operands as the decode does (scores
// S^T = K Q^T, values O^T += V^T P^T; heads are columns), from a list instead of a table's row: 64
// entries at a time become pool offsets, those that name no visible block dropped.
//
// A product has 16 columns and a group often fewer heads, so the heads stand in the columns
// kWays = 2 or 4 times over (g <= 8, g <= 4), and column (way w, head h) goes on with the scores of
// blocks w, w + kWays, ... alone. Every lane's exponentials are then of use (4 per lane and step instead
// of 16 at g <= 4), the ways share a maximum, and their sums meet at the end of the wave's share.
//
// The value product takes bf16, and a weight rounded to it would be off by up to 2^-8 of itself, which
// stands beside the output's own rounding. So a weight goes in two parts, itself rounded and what that
// left over, off by at most 2^-16 together. The second part costs no product where there are several
// ways: it stands in the next way's column, whose weights for the block would be zeros (kWays 1 takes a
// second product).
//
// A column's maximum is only brought up to date when a score passes it by 2^kSlack: until then
// weights may reach 2^kSlack, which costs no precision (32-bit sums, and bf16 has the same relative step
// everywhere), and most steps need no lane exchange and no rescaling.
//
// A zero weight is no mask for a value that is not finite: 0 x inf is NaN, in the columns of the ways
// that the value is not for, two parts of either sign make NaN of it too, and weights of 2^kSlack
// may carry large values past the 32-bit range. A wave whose sums are not finite takes its share again
// with one way, weights in one part and maxima always up to date (sparse_share), as the decode does: an
// infinite value then makes its dim infinite, and a finite one does not, whatever the number of heads.
// Sums that are finite cost one look per wave.
#include <math.h>

#include "decode_impl.h"
#include "launch.h"
#include "wave_utils.h"

namespace pkv {
namespace {

using dec::finite_max;

constexpr int kStep = 4;         // blocks per step
constexpr float kSlack = 8.f;    // (base 2)
constexpr int kMergeWaves = 4;
constexpr int kParts = 4;        // waves that share an item where items are few
constexpr int kXcds = 8;         // workgroups go to the chip's XCDs in turn

// Odd rows (of 16 lanes) of a and even rows of b change places.
__device__ __forceinline__ u32x2 swap_rows(uint32_t a, uint32_t b) {
#if __HIP_DEVICE_COMPILE__
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  return u32x2{r[0], r[1]};
#else
  return u32x2{a, b};
#endif
}

// One wave's share: entries [e0, e1) of a list. Leaves, summed over the ways, the unnormalised output
// (lane (col, grp) holds dims 16 db + 4 grp + 0..3 of head col % (16 / kWays)), the maximum (base 2)
// and the weight sum.
template <int D, int kWays, bool kTwoParts>
__device__ __forceinline__ void sparse_range(const SparseArgs& a, const bf16x8 (&qf)[D / 32],
                                             const int32_t* __restrict__ list,
                                             const int32_t* __restrict__ table, const int kvh,
                                             const int len, const int e0, const int e1,
                                             f32x4 (&acc_out)[D / 16], float& m_out,
                                             float& l_out) {
  constexpr int KK = D / 32, DB = D / 16, SLAB = D * kBlockSize;
  constexpr int SLAB_BYTES = SLAB * 2;
  constexpr int kMine = kStep / kWays;  // blocks per step whose scores a column goes on with
  constexpr float kPast = kTwoParts ? kSlack : 0.f;  // (the other form takes sums that overflow, too)
  const int lane = threadIdx.x & 63;
  const int col = lane & 15, grp = lane >> 4;
  const int way = col / (16 / kWays);
  const int n = len > 0 ? min((len - 1) / kBlockSize + 1, a.max_blocks) : 0;  // the row's blocks
  const size_t head_off = (size_t)kvh * SLAB;
  f32x4 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, lpart = 0.f;

  auto entry = [&](int e) { return e + lane < e1 ? list[e + lane] : -1; };
  auto lookup = [&](int b) { return b >= 0 && b < n ? table[b] : -1; };
  int b = entry(e0), b_next = entry(e0 + 64);
  int id = lookup(b);
  for (int e = e0; e < e1; e += 64) {
    const int id_next = lookup(b_next);
    const int b_then = entry(e + 128);
    // 64 entries: pool block and filled slots, the visible ones moved to the front lanes
    const bool live = id >= 0 && id < a.num_blocks;
    int keys = live ? min(len - b * kBlockSize, kBlockSize) : 0;
    int blk = live ? id : 0;  // (a stand-in, read and masked)
    const uint64_t mask = __builtin_amdgcn_ballot_w64(live);
    const int count = __builtin_popcountll(mask);
    const uint64_t below = (1ull << lane) - 1;
    const int to = live ? __builtin_popcountll(mask & below)
                        : count + __builtin_popcountll(~mask & below);
    blk = __builtin_amdgcn_ds_permute(to * 4, blk);
    keys = __builtin_amdgcn_ds_permute(to * 4, keys);
    const uint64_t partial = __builtin_amdgcn_ballot_w64(keys < kBlockSize);
    b = b_next;
    id = id_next;
    b_next = b_then;
    if (count == 0) continue;

    u32x4 k[kStep][KK];
    u32x4 v[kStep / 2][DB];
    auto slab = [&](int s) {  // (steps end within 64 entries: kStep divides 64)
      return (size_t)__builtin_amdgcn_readlane(blk, s) * a.hkv * SLAB + head_off;
    };
    auto load_k = [&](int s) {
#pragma unroll
      for (int i = 0; i < kStep; ++i) {
        const uint16_t* base = a.k_cache + slab(s + i);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
          k[i][kk] = buf_ld16(base, SLAB_BYTES, ((grp + 4 * kk) * kBlockSize + col) * 16);
      }
    };
    auto load_v = [&](int s) {
#pragma unroll
      for (int i = 0; i < kStep / 2; ++i) {
        const size_t even = slab(s + 2 * i), odd = slab(s + 2 * i + 1);
        const uint16_t* base = a.v_cache + ((grp & 1) ? odd : even) + col * kBlockSize + (grp >> 1) * 8;
#pragma unroll
        for (int db = 0; db < DB; ++db) v[i][db] = ld16(base + db * 16 * kBlockSize);
      }
    };
    load_k(0);
    load_v(0);
    for (int s = 0; s < count; s += kStep) {
      f32x4 st[kStep];
#pragma unroll
      for (int i = 0; i < kStep; ++i) {
        st[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) st[i] = mfma16(as_bf16x8(k[i][kk]), qf[kk], st[i]);
      }
      const bool more = s + kStep < count;
      if (more) load_k(s + kStep);  // (in flight through the rest of this step)
      const bool cut = (partial >> s & ((1u << kStep) - 1)) != 0;
      if (cut) {
#pragma unroll
        for (int i = 0; i < kStep; ++i) {
          const int filled = __builtin_amdgcn_readlane(keys, s + i);
#pragma unroll
          for (int r = 0; r < 4; ++r) st[i][r] = 4 * grp + r < filled ? st[i][r] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < kStep / 2; ++i) {
          const int even = __builtin_amdgcn_readlane(keys, s + 2 * i);
          const int odd = __builtin_amdgcn_readlane(keys, s + 2 * i + 1);
          const int filled = ((grp & 1) ? odd : even) - 8 * (grp >> 1);
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const u32x2 lo = dec::mask_v4(u32x2{v[i][db][0], v[i][db][1]}, 0, filled);
            const u32x2 hi = dec::mask_v4(u32x2{v[i][db][2], v[i][db][3]}, 4, filled);
            v[i][db] = u32x4{lo[0], lo[1], hi[0], hi[1]};
          }
        }
      }
      // lane holds keys 4 grp + r of its way's blocks
      float sv[kMine][4];
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float x = st[j * kWays][r];
#pragma unroll
          for (int w = 1; w < kWays; ++w) x = way == w ? st[j * kWays + w][r] : x;
          sv[j][r] = x;
          mx = fmaxf(mx, x);
        }
      }
      mx *= a.scale_log2;
      if (__builtin_amdgcn_ballot_w64(mx > m + kPast) != 0) {
        const float m_new = fmaxf(m, ways_max<kWays>(dec::wave_max16(mx)));
        const float alpha = fast_exp2(m - finite_max(m_new));
        m = m_new;
        lpart *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[db][r] *= alpha;
        }
      }
      const float m_sub = finite_max(m);
      constexpr int kProducts = kWays == 1 && kTwoParts ? 2 : 1;
      uint32_t p[kProducts][kStep][2];
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = fast_exp2(fmaf(sv[j][r], a.scale_log2, -m_sub));
          lpart += x[r];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint32_t first, second;
          two_parts(x[2 * e], x[2 * e + 1], first, second);
          if constexpr (kWays == 1) {
            p[0][j][e] = first;
            if constexpr (kTwoParts) p[1][j][e] = second;
          } else {
            // (the second part of the way before, from its columns)
            second = dpp<kWays == 4 ? kRor4 : kRor8>(second);
#pragma unroll
            for (int w = 0; w < kWays; ++w)
              p[0][j * kWays + w][e] = way == w ? first : way == (w + 1) % kWays ? second : 0u;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kProducts; ++k) {
#pragma unroll
        for (int i = 0; i < kStep; i += 2) {
          const u32x2 x = swap_rows(p[k][i][0], p[k][i + 1][0]);
          const u32x2 y = swap_rows(p[k][i][1], p[k][i + 1][1]);
          const u32x4 pb = {x[0], y[0], x[1], y[1]};
#pragma unroll
          for (int db = 0; db < DB; ++db)
            acc[db] = mfma16(as_bf16x8(v[i / 2][db]), as_bf16x8(pb), acc[db]);
        }
      }
      if (more) load_v(s + kStep);
    }
  }
  l_out = ways_sum<kWays>(dec::wave_sum16(lpart));
  m_out = m;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
#pragma unroll
    for (int r = 0; r < 4; ++r) acc_out[db][r] = ways_sum<kWays>(acc[db][r]);
  }
}

// A row's part in a launch: which list and table, how many keys it sees.
struct SparseRow {
  int64_t item, row;
  int kvh, seq, len;
};
__device__ __forceinline__ bool sparse_row(const SparseArgs& a, int64_t item, SparseRow& r) {
  if (a.xcd_items > 0) {
    const int64_t k = (item % kXcds) * a.xcd_items + item / kXcds;
    if (k >= a.rows * a.hkv) return false;
    r.kvh = (int)(k / a.rows);
    r.row = k % a.rows;
  } else {
    r.row = item / a.hkv;
    r.kvh = (int)(item % a.hkv);
  }
  r.item = r.row * a.hkv + r.kvh;
  r.seq = a.row_seq != nullptr ? a.row_seq[r.row] : (int)r.row;
  if (r.seq < 0 || r.seq >= a.num_seqs) return false;  // a padding row
  r.len = max(a.row_lens[r.row], 0);
  return true;
}
// The query operand, the heads kWays times over (zeros past the group's heads).
template <int D, int kWays>
__device__ __forceinline__ void sparse_load_q(const SparseArgs& a, const SparseRow& r, int g,
                                              bf16x8 (&qf)[D / 32]) {
  const int lane = threadIdx.x & 63, h = (lane & 15) % (16 / kWays), grp = lane >> 4;
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if (h < g) v = ld16(a.q + ((size_t)r.row * a.hq + r.kvh * g + h) * D + kk * 32 + grp * 8);
    qf[kk] = as_bf16x8(v);
  }
}

// The wave's share, infinities and NaN in it as the sums' definition has them.
template <int D, int kWays>
__device__ __forceinline__ void sparse_share(const SparseArgs& a, const SparseRow& r,
                                             const bf16x8 (&qf)[D / 32], const int e0,
                                             const int e1, f32x4 (&acc)[D / 16], float& m,
                                             float& l) {
  const int32_t* list = a.sel + r.item * a.blocks;
  const int32_t* table = a.tables + (size_t)r.seq * a.max_blocks;
  sparse_range<D, kWays, true>(a, qf, list, table, r.kvh, r.len, e0, e1, acc, m, l);
  float odd = 0.f;  // NaN if a sum is not finite
#pragma unroll
  for (int db = 0; db < D / 16; ++db) {
#pragma unroll
    for (int e = 0; e < 4; ++e) odd = fmaf(acc[db][e], 0.f, odd);
  }
  if (__builtin_amdgcn_ballot_w64(odd != odd) != 0)
    sparse_range<D, 1, false>(a, qf, list, table, r.kvh, r.len, e0, e1, acc, m, l);
}

// One wave per (row, kv head).
template <int D, int kWays>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void sparse_wave_kernel(const SparseArgs a) {
  constexpr int DB = D / 16;
  SparseRow r;
  if (!sparse_row(a, blockIdx.x, r)) return;
  const int g = a.hq / a.hkv;
  bf16x8 qf[D / 32];
  sparse_load_q<D, kWays>(a, r, g, qf);
  f32x4 acc[DB];
  float m, l;
  sparse_share<D, kWays>(a, r, qf, 0, a.blocks, acc, m, l);
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int h = col % (16 / kWays), way = col / (16 / kWays);
  if (h >= g) return;
  const size_t o = (size_t)r.row * a.hq + r.kvh * g + h;
  // no weight (no visible key, or scores of -infinity alone): zeros, whatever the sums hold
  const float inv = 1.f / l;
  uint16_t* dst = a.out + o * D;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    if (db % kWays != way) continue;  // (each way stores its part)
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = l == 0.f ? 0.f : acc[db][e] * inv;
    st8(dst + db * 16 + 4 * grp, u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])});
  }
  if (a.lse != nullptr && lane < 16 / kWays) a.lse[o] = (m + log2f(l)) * kLn2;
}

// kParts waves per (row, kv head, split): each takes an equal share of the split's entries, and the
// shares meet in LDS. With several splits, the results are partial ones for the merge below.
template <int D, int kWays>
__global__ __launch_bounds__(64 * kParts) __attribute__((amdgpu_waves_per_eu(2, 2)))
void sparse_group_kernel(const SparseArgs a) {
  constexpr int DB = D / 16;
  __shared__ __align__(16) dec::DecodeSmem<D, kParts> sm;
  SparseRow r;
  if (!sparse_row(a, blockIdx.x / a.splits, r)) return;  // (workgroup-uniform)
  const int split = (int)(blockIdx.x % a.splits);
  const int g = a.hq / a.hkv;
  const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int e0 = min(split * a.split_entries, a.blocks);
  const int e1 = min(e0 + a.split_entries, a.blocks);
  const int share = ((e1 - e0 + kParts - 1) / kParts + kStep - 1) / kStep * kStep;
  const int s0 = min(e0 + wave * share, e1), s1 = min(s0 + share, e1);
  bf16x8 qf[D / 32];
  sparse_load_q<D, kWays>(a, r, g, qf);
  f32x4 acc[DB];
  float m, l;
  sparse_share<D, kWays>(a, r, qf, s0, s1, acc, m, l);
  const int hcol = col % (16 / kWays), way = col / (16 / kWays);
  if (hcol < g) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
      if (db % kWays == way)
        st16(&sm.o[wave][hcol][db * 16 + 4 * grp], __builtin_bit_cast(u32x4, acc[db]));
    if (lane < 16 / kWays) {
      sm.m[wave][hcol] = m;
      sm.l[wave][hcol] = l;
    }
  }
  __syncthreads();
  for (int u = threadIdx.x; u < g * (D / 4); u += 64 * kParts) {  // one thread per (head, 4 dims)
    const int h = u / (D / 4), d = (u % (D / 4)) * 4;
    float mx = -INFINITY;
#pragma unroll
    for (int s = 0; s < kParts; ++s) mx = fmaxf(mx, sm.m[s][h]);
    float den = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
      const float w = fast_exp2(sm.m[s][h] - finite_max(mx));
      den += w * sm.l[s][h];
      const f32x4 x = __builtin_bit_cast(f32x4, ld16(&sm.o[s][h][d]));
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += w * x[e];
    }
    const size_t row = (size_t)r.row * a.hq + r.kvh * g + h;
    if (a.splits == 1) {
      const float inv = 1.f / den;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = den == 0.f ? 0.f : o[e] * inv;
      st8(a.out + row * D + d, u32x2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])});
      if (a.lse != nullptr && d == 0) a.lse[row] = (mx + log2f(den)) * kLn2;
    } else {
      const size_t slot = row * a.splits + split;
      st16(a.ws_o + slot * D + d, __builtin_bit_cast(u32x4, o));
      if (d == 0) {
        a.ws_ml[slot * 2] = mx;
        a.ws_ml[slot * 2 + 1] = den;
      }
    }
  }
}

// One wave per (row, query head): the splits' partial results by their log-sum-exp weights.
template <int D>
__global__ __launch_bounds__(64 * kMergeWaves) void sparse_merge_kernel(const SparseArgs a) {
  constexpr int PER = D / 64;
  const int64_t item = (int64_t)blockIdx.x * kMergeWaves + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (item >= a.rows * a.hq) return;
  const int64_t row = item / a.hq;
  const int seq = a.row_seq != nullptr ? a.row_seq[row] : (int)row;
  if (seq < 0 || seq >= a.num_seqs) return;
  const float* ml = a.ws_ml + (size_t)item * a.splits * 2;
  const float* src = a.ws_o + (size_t)item * a.splits * D + lane * PER;
  const bool mine = lane < a.splits;  // (at most 64 splits)
  const float m = mine ? ml[lane * 2] : -INFINITY;
  const float l = mine ? ml[lane * 2 + 1] : 0.f;
  float top = m;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float w = mine ? fast_exp2(m - finite_max(top)) : 0.f;
  float den = w * l;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) den += __shfl_xor(den, o);
  float o[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = 0.f;
  for (int s = 0; s < a.splits; s += 8) add_partials<D>(src, w, s, a.splits, o);
  const float inv = 1.f / den;
  uint16_t* dst = a.out + (size_t)item * D + lane * PER;
#pragma unroll
  for (int e = 0; e < PER; ++e) o[e] = den == 0.f ? 0.f : o[e] * inv;
  if constexpr (PER == 2) {
    *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(o[0], o[1]);
  } else {
    dst[0] = (uint16_t)(pack_bf16x2(o[0], 0.f) & 0xFFFFu);
  }
  if (a.lse != nullptr && lane == 0) a.lse[item] = (top + log2f(den)) * kLn2;
}

// How a call is cut: host arithmetic on its sizes alone (D = 128, 8 kv heads; us).
struct SparseCut {
  int parts;          // waves per (row, kv head, split)
  int splits;         // workgroups per (row, kv head)
  int split_entries;  // list entries of each
};
SparseCut sparse_cut(int64_t items, int32_t blocks) {
  SparseCut c{1, 1, blocks};
  // Four waves share an item while there are too few to fill the chip with one wave each, if each
  // share is a step of its own at least: 64 items of 32 blocks 6.9 against 9.9, of 128 16.9 against
  // 34.3, 256 of 128 43.6 and 47.0; but 64 of 4 blocks 5.2 and 4.7, 512 of 32 25.2 and 24.9, 1024 of
  // 128 187 and 169. (Eight waves: 7.3, 17.1, 44.3; never ahead by more than the noise.)
  if (items < 512 && blocks > 2 * kStep) c.parts = kParts;
  // Splits across workgroups fill the chip where items are few, for partial results and a merge
  // launch (about 3 us): long lists only, the longer the more items there are. 8 items of 128 blocks
  // 8.7 in eight splits against 11.8, of 512 13.7 against 42.5; 32 of 128 11.0 and 15.0; 64 of 512
  // 48.7 (four) and 73.9; but 8 of 64 8.5 and 8.4, 64 of 128 18.3 and 16.9, 128 of 256 46.1 and 45.0.
  if (blocks >= 96 && blocks >= 4 * items && items <= 128) {
    const int most = std::min((int)(256 / items), blocks / 16);
    c.split_entries = (blocks + most - 1) / most;
    c.split_entries = (c.split_entries + kParts * kStep - 1) / (kParts * kStep) * (kParts * kStep);
    c.splits = (blocks + c.split_entries - 1) / c.split_entries;
    if (c.splits > 64) {  // (a lane each in the merge)
      c.split_entries = (blocks + 63) / 64;
      c.splits = (blocks + c.split_entries - 1) / c.split_entries;
    }
  }
  return c;
}

template <int D, int kWays>
hipError_t launch_cut(const SparseArgs& a, const SparseCut& c, int64_t items, hipStream_t stream) {
  if (a.xcd_items > 0) items = kXcds * a.xcd_items;
  auto* kern = c.parts == 1 ? sparse_wave_kernel<D, kWays> : sparse_group_kernel<D, kWays>;
  hipLaunchKernelGGL(kern, dim3((unsigned)(items * c.splits)), dim3(64 * c.parts), 0, stream, a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || c.splits == 1) return err;
  const int64_t rows = a.rows * a.hq;
  hipLaunchKernelGGL(sparse_merge_kernel<D>,
                     dim3((unsigned)((rows + kMergeWaves - 1) / kMergeWaves)),
                     dim3(64 * kMergeWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t sparse_workspace_bytes(int64_t items, int32_t g, int32_t head_dim, int32_t blocks) {
  const SparseCut c = sparse_cut(items, blocks);
  if (c.splits == 1) return 0;
  return (size_t)items * g * c.splits * (head_dim + 2) * sizeof(float);
}

hipError_t launch_sparse_attention(SparseArgs a, int head_dim, void* workspace,
                                   hipStream_t stream) {
  const int64_t items = a.rows * a.hkv;
  const SparseCut c = sparse_cut(items, a.blocks);
  // Rows of longer suffixes share their sequences' keys: each XCD takes a run of rows of one kv head
  // after the other, so that its L2 holds few heads' keys at a time (1525 rows of five sequences, 63
  // random blocks each, inputs changing: 20/5 heads 173 us against 346 with items in order, 16/16 532 and
  // 678, 16/4 of 64 dims 65.8 and 67.3; with 8 kv heads an order of items gives each XCD one head as
  // well: 32/8 259 both ways).
  a.xcd_items = a.row_seq != nullptr ? (items + kXcds - 1) / kXcds : 0;
  a.splits = c.splits;
  a.split_entries = c.split_entries;
  a.ws_o = static_cast<float*>(workspace);
  a.ws_ml = a.ws_o + (size_t)a.rows * a.hq * c.splits * head_dim;
  const int g = a.hq / a.hkv;
  if (head_dim == 128)
    return g <= 4   ? launch_cut<128, 4>(a, c, items, stream)
           : g <= 8 ? launch_cut<128, 2>(a, c, items, stream)
                    : launch_cut<128, 1>(a, c, items, stream);
  return g <= 4   ? launch_cut<64, 4>(a, c, items, stream)
         : g <= 8 ? launch_cut<64, 2>(a, c, items, stream)
                  : launch_cut<64, 1>(a, c, items, stream);
}

}  // namespace pkv
